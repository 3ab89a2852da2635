// Dropout from a counter-based generator, with the residual's addition; the mask is never stored.
//
//   u_i = 16 bits of Philox4x32-10 (Salmon, Moraes, Dror, Shaw: Parallel random numbers: as easy as 1, 2, 3; 2011),
//   y_i = res_i + (u_i >= t ? x_i 65536 / (65536 - t) : 0),   t = drop probability in units of 2^-16
//
// One block of the generator gives eight elements their 16 bits each, so that ten rounds of two 32-bit multiplications are
// shared by eight values and the kernel stays bound by memory: x, res and y once each.  Eight elements per thread and step
// are one 16-byte vector of bf16 or two of fp32.  Measured at 33.5 M values: bf16 37 us with a residual (5.5 TB/s), 29 us
// without (4.7 TB/s, the generator takes two thirds of the issue slots); fp32 61 and 44 us (6.6 and 6.1 TB/s).
#include <algorithm>

#include "common.cuh"
#include "lm_ops.h"

namespace ddg {

namespace {

// N blocks of the generator side by side: they share the keys' increments.
template <int N> __device__ __forceinline__ void philox(const unsigned long long (&at)[N], uint32_t layer, uint32_t k0, uint32_t k1, uint32_t (&w)[N][4]) {
#pragma unroll
    for (int u = 0; u < N; ++u) { w[u][0] = (uint32_t)at[u]; w[u][1] = (uint32_t)(at[u] >> 32); w[u][2] = layer; w[u][3] = 0; }
#pragma unroll
    for (int r = 0; r < 10; ++r) {
#pragma unroll
        for (int u = 0; u < N; ++u) {
            const uint64_t p = (uint64_t)w[u][0] * 0xD2511F53u, q = (uint64_t)w[u][2] * 0xCD9E8D57u;
            w[u][0] = (uint32_t)(q >> 32) ^ w[u][1] ^ k0;
            w[u][2] = (uint32_t)(p >> 32) ^ w[u][3] ^ k1;
            w[u][1] = (uint32_t)q;
            w[u][3] = (uint32_t)p;
        }
        k0 += 0x9E3779B9u;
        k1 += 0xBB67AE85u;
    }
}

// Eight elements as they lie in memory: 16 bytes of bf16, 32 of fp32.
template <typename T> struct Raw8 {
    uint4 q[sizeof(T) / 2];
    __device__ __forceinline__ void load(const T *p) {
#pragma unroll
        for (int i = 0; i < (int)sizeof(T) / 2; ++i) q[i] = reinterpret_cast<const uint4 *>(p)[i];
    }
    __device__ __forceinline__ void store(T *p) const {
#pragma unroll
        for (int i = 0; i < (int)sizeof(T) / 2; ++i) reinterpret_cast<uint4 *>(p)[i] = q[i];
    }
    __device__ __forceinline__ T *elems() { return reinterpret_cast<T *>(q); }
};

// y may be x or res.  vec: every tensor starts on a 16-byte boundary.  A thread takes kUnroll blocks at a time; their loads
// are in flight while it computes the generator's.
constexpr int kUnroll = 2;
constexpr size_t kGrid = 148 * 16;
template <typename T, bool RES>
__global__ void __launch_bounds__(256) dropout_kernel(const T *x, const T *res, T *y, const unsigned long long *__restrict__ rng, size_t n, unsigned threshold,
                                                      float scale, unsigned layer, int vec) {
    pdl_launch();
    pdl_wait();
    const unsigned long long key = rng[0], start = rng[1];
    const size_t blocks = (n + 7) / 8, whole = vec ? n / 8 : 0, stride = (size_t)gridDim.x * 256;
    const bool all = threshold > 65535u;  // p = 1: nothing is kept (the comparison below has 16 bits)
    for (size_t i0 = (size_t)blockIdx.x * 256 + threadIdx.x; i0 < blocks; i0 += stride * kUnroll) {
        Raw8<T> a[kUnroll], b[kUnroll];
#pragma unroll
        for (int u = 0; u < kUnroll; ++u) {
            const size_t i = i0 + u * stride;
            if (i < whole) {
                a[u].load(x + i * 8);
                if (RES) b[u].load(res + i * 8);
            } else if (i < blocks) {
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    a[u].elems()[j] = i * 8 + j < n ? x[i * 8 + j] : from_f<T>(0.f);
                    if (RES) b[u].elems()[j] = i * 8 + j < n ? res[i * 8 + j] : from_f<T>(0.f);
                }
            }
        }
        unsigned long long at[kUnroll];
        uint32_t w[kUnroll][4];
#pragma unroll
        for (int u = 0; u < kUnroll; ++u) at[u] = start + i0 + u * stride;
        philox(at, layer, (uint32_t)key, (uint32_t)(key >> 32), w);
#pragma unroll
        for (int u = 0; u < kUnroll; ++u) {
            const size_t i = i0 + u * stride;
            if (i >= blocks) break;
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                // 16 bits against the threshold, in the upper half of a word: what stands below them does not matter
                const bool keep = ((j & 1) ? w[u][j / 2] : w[u][j / 2] << 16) >= threshold << 16 && !all;
                const float v = keep ? to_f(a[u].elems()[j]) : 0.f;  // a dropped infinity or NaN is zero
                a[u].elems()[j] = from_f<T>(RES ? fmaf(v, scale, to_f(b[u].elems()[j])) : v * scale);
            }
            if (i < whole) {
                a[u].store(y + i * 8);
            } else {
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    if (i * 8 + j < n) y[i * 8 + j] = a[u].elems()[j];
            }
        }
    }
}

template <typename T>
void dropout_as(const void *x, const void *res, void *y, const unsigned long long *rng, size_t n, unsigned threshold, float scale, unsigned layer, int vec, int grid,
                const Launch &s) {
    if (res) launch_k(dropout_kernel<T, true>, grid, 256, 0, s, (const T *)x, (const T *)res, (T *)y, rng, n, threshold, scale, layer, vec);
    else launch_k(dropout_kernel<T, false>, grid, 256, 0, s, (const T *)x, (const T *)res, (T *)y, rng, n, threshold, scale, layer, vec);
}

}  // namespace

int launch_dropout(int prec, const void *x, const void *res, void *y, const unsigned long long *rng, size_t n, unsigned threshold, unsigned layer, Launch s) {
    const int vec = ((reinterpret_cast<uintptr_t>(x) | reinterpret_cast<uintptr_t>(res) | reinterpret_cast<uintptr_t>(y)) & 15) == 0;
    const float scale = threshold < 65536u ? (float)(65536.0 / (65536.0 - threshold)) : 0.f;
    const int grid = (int)std::min<size_t>(((n + 7) / 8 + 255) / 256, kGrid);
    if (prec == P_BF16) dropout_as<bf16>(x, res, y, rng, n, threshold, scale, layer, vec, grid, s);
    else dropout_as<float>(x, res, y, rng, n, threshold, scale, layer, vec, grid, s);
    return 1;
}

}  // namespace ddg

// Dropout from a counter-based generator, with the residual's addition; the mask is never stored.
//
//   u_i = 16 bits of Philox4x32-10 (Salmon, Moraes, Dror, Shaw: Parallel random numbers: as easy as 1, 2, 3; 2011),
//   y_i = res_i + (u_i >= t ? x_i 65536 / (65536 - t) : 0),   t = drop probability in units of 2^-16
//
// One block of the generator gives eight elements their 16 bits each, so that ten rounds of two 32-bit multiplications are
// shared by eight values and the kernel stays bound by memory: x, res and y once each.  Eight elements per thread and step
// are one 16-byte vector of bf16 or two of fp32.
#include <algorithm>

#include "common.cuh"
#include "lm_ops.h"

namespace ddg {

namespace {

__device__ __forceinline__ uint4 philox(uint32_t c0, uint32_t c1, uint32_t c2, uint32_t k0, uint32_t k1) {
    uint32_t c3 = 0;
#pragma unroll
    for (int r = 0; r < 10; ++r) {
        const uint64_t p = (uint64_t)c0 * 0xD2511F53u, q = (uint64_t)c2 * 0xCD9E8D57u;
        c0 = (uint32_t)(q >> 32) ^ c1 ^ k0;
        c2 = (uint32_t)(p >> 32) ^ c3 ^ k1;
        c1 = (uint32_t)q;
        c3 = (uint32_t)p;
        k0 += 0x9E3779B9u;
        k1 += 0xBB67AE85u;
    }
    return make_uint4(c0, c1, c2, c3);
}

template <typename T> __device__ __forceinline__ void load8(const T *p, float (&v)[8]) {
    if (sizeof(T) == 2) {
        load_f<T, 8>(p, v);
    } else {
        load_f<T, 4>(p, reinterpret_cast<float(&)[4]>(v[0]));
        load_f<T, 4>(p + 4, reinterpret_cast<float(&)[4]>(v[4]));
    }
}
template <typename T> __device__ __forceinline__ void store8(T *p, const float (&v)[8]) {
    if (sizeof(T) == 2) {
        store_f<T, 8>(p, v);
    } else {
        store_f<T, 4>(p, reinterpret_cast<const float(&)[4]>(v[0]));
        store_f<T, 4>(p + 4, reinterpret_cast<const float(&)[4]>(v[4]));
    }
}

// y may be x or res.  vec: every tensor starts on a 16-byte boundary.
template <typename T>
__global__ void __launch_bounds__(256) dropout_kernel(const T *x, const T *res, T *y, const unsigned long long *__restrict__ rng, size_t n, unsigned threshold,
                                                      float scale, unsigned layer, int vec) {
    pdl_launch();
    pdl_wait();
    const unsigned long long key = rng[0], start = rng[1];
    const size_t blocks = (n + 7) / 8;
    for (size_t i = (size_t)blockIdx.x * 256 + threadIdx.x; i < blocks; i += (size_t)gridDim.x * 256) {
        const unsigned long long at = start + i;
        const uint4 u = philox((uint32_t)at, (uint32_t)(at >> 32), layer, (uint32_t)key, (uint32_t)(key >> 32));
        const uint32_t w[4] = {u.x, u.y, u.z, u.w};
        const bool whole = vec && i * 8 + 8 <= n;
        float v[8], b[8];
        if (whole) {
            load8(x + i * 8, v);
            if (res) load8(res + i * 8, b);
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                v[j] = i * 8 + j < n ? to_f(x[i * 8 + j]) : 0.f;
                b[j] = res && i * 8 + j < n ? to_f(res[i * 8 + j]) : 0.f;
            }
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const uint32_t r = (j & 1) ? w[j / 2] >> 16 : w[j / 2] & 0xffffu;
            v[j] = r >= threshold ? v[j] * scale : 0.f;  // a dropped infinity or NaN is zero
            if (res) v[j] += b[j];
        }
        if (whole) {
            store8(y + i * 8, v);
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j)
                if (i * 8 + j < n) y[i * 8 + j] = from_f<T>(v[j]);
        }
    }
}

}  // namespace

int launch_dropout(int prec, const void *x, const void *res, void *y, const unsigned long long *rng, size_t n, unsigned threshold, unsigned layer, Launch s) {
    const int vec = ((reinterpret_cast<uintptr_t>(x) | reinterpret_cast<uintptr_t>(res) | reinterpret_cast<uintptr_t>(y)) & 15) == 0;
    const float scale = threshold < 65536u ? (float)(65536.0 / (65536.0 - threshold)) : 0.f;
    const int grid = (int)std::min<size_t>(((n + 7) / 8 + 255) / 256, 148 * 16);
    if (prec == P_BF16)
        launch_k(dropout_kernel<bf16>, grid, 256, 0, s, (const bf16 *)x, (const bf16 *)res, (bf16 *)y, rng, n, threshold, scale, layer, vec);
    else
        launch_k(dropout_kernel<float>, grid, 256, 0, s, (const float *)x, (const float *)res, (float *)y, rng, n, threshold, scale, layer, vec);
    return 1;
}

}  // namespace ddg

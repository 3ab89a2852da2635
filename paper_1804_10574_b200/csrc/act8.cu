// Activation checkpoints in 8 bits: rows of a tensor to codes with a scale per row, and back (act8.cuh has the formulas).
//
// Bound by memory: packing reads a row once and writes a quarter or half of its bytes; the row stays in its threads'
// registers between the maximum and the codes.  Rows wider than that (16384 values) are read twice.
#include <algorithm>

#include "act8.cuh"
#include "common.cuh"
#include "lm_ops.h"
#include "row_io.cuh"

namespace ddg {

namespace {

__device__ __forceinline__ uint32_t magnitude_bits(float v) { return __float_as_uint(v) & 0x7fffffffu; }

__device__ __forceinline__ uint32_t row_max_bits(uint32_t v, bool one_warp, uint32_t *red) {
    v = __reduce_max_sync(0xffffffffu, v);
    if (one_warp) return v;
    const int nw = blockDim.x >> 5, lane = threadIdx.x & 31;
    if (lane == 0) red[threadIdx.x >> 5] = v;
    __syncthreads();
    return __reduce_max_sync(0xffffffffu, lane < nw ? red[lane] : 0u);
}

template <typename T, int VEC, int ITER>
__global__ void __launch_bounds__(rms_max_threads(VEC, ITER)) act8_pack_kernel(const T *__restrict__ x, int8_t *__restrict__ q, float *__restrict__ scale, int rows, int C, int pitch, int tpr) {
    __shared__ uint32_t red[32];
    pdl_launch();
    pdl_wait();
    const bool one_warp = tpr == 32;
    const int t = one_warp ? (threadIdx.x & 31) : threadIdx.x;
    const int row = one_warp ? blockIdx.x * (blockDim.x >> 5) + (threadIdx.x >> 5) : blockIdx.x;
    if (row >= rows) return;  // whole warps, and only where a row is one warp's
    const T *from = x + (size_t)row * C;
    int8_t *to = q + (size_t)row * pitch;
    float v[ITER][VEC];
    uint32_t top = 0;
#pragma unroll
    for (int i = 0; i < ITER; ++i) {
        const int c = (i * tpr + t) * VEC;
        if (c < C) {
            load_f<T, VEC>(from + c, v[i]);
#pragma unroll
            for (int j = 0; j < VEC; ++j) top = max(top, magnitude_bits(v[i][j]));
        }
    }
    top = row_max_bits(top, one_warp, red);
    float s;
    const Act8Row r = act8_row(top, s);
    if (t == 0) scale[row] = s;
#pragma unroll
    for (int i = 0; i < ITER; ++i) {
        const int c = (i * tpr + t) * VEC;
        if (c < C) {
            act8_store<sizeof(T) == 2, VEC>(to + c, v[i], r);
        }
    }
    for (int c = C + t; c < pitch; c += tpr) to[c] = 0;
}

// Rows of more values than a block's registers hold: read twice, the second time out of the L2.
template <typename T>
__global__ void __launch_bounds__(1024) act8_pack_wide_kernel(const T *__restrict__ x, int8_t *__restrict__ q, float *__restrict__ scale, int C, int pitch) {
    __shared__ uint32_t red[32];
    pdl_launch();
    pdl_wait();
    const T *from = x + (size_t)blockIdx.x * C;
    int8_t *to = q + (size_t)blockIdx.x * pitch;
    uint32_t top = 0;
#pragma unroll 8
    for (int c = threadIdx.x; c < C; c += 1024) top = max(top, magnitude_bits(to_f(from[c])));
    top = row_max_bits(top, false, red);
    float s;
    const Act8Row r = act8_row(top, s);
    if (threadIdx.x == 0) scale[blockIdx.x] = s;
#pragma unroll 4
    for (int c = threadIdx.x; c < pitch; c += 1024) to[c] = c < C ? (int8_t)act8_code(to_f(from[c]), r) : (int8_t)0;
}

// 16 codes of a row per thread.
template <typename T>
__global__ void __launch_bounds__(256) act8_unpack_kernel(const int8_t *__restrict__ q, const float *__restrict__ scale, T *__restrict__ x, size_t units, int C, int pitch, int vec) {
    pdl_launch();
    pdl_wait();
    const unsigned per_row = pitch / 16;
    for (size_t i = (size_t)blockIdx.x * 256 + threadIdx.x; i < units; i += (size_t)gridDim.x * 256) {
        const size_t row = units <= 0xffffffffu ? (unsigned)i / per_row : i / per_row;
        const int c = (int)(i - row * per_row) * 16;
        const uint4 w = *reinterpret_cast<const uint4 *>(q + row * pitch + c);
        const float s = scale[row];
        const uint32_t word[4] = {w.x, w.y, w.z, w.w};
        T *to = x + row * C + c;
        float v[16];
#pragma unroll
        for (int j = 0; j < 16; ++j) v[j] = (float)(int8_t)(word[j / 4] >> (8 * (j % 4))) * s;
        constexpr int N = Vec16<T>::N;
        if (vec) {
#pragma unroll
            for (int j = 0; j < 16; j += N)
                if (c + j < C) store_f<T, N>(to + j, reinterpret_cast<const float(&)[N]>(v[j]));
        } else {
#pragma unroll
            for (int j = 0; j < 16; ++j)
                if (c + j < C) to[j] = from_f<T>(v[j]);
        }
    }
}

template <typename T, int VEC> int pack_as(const void *x, void *q, float *scale, int rows, int C, const Launch &s) {
    const int pitch = act8_pitch(C);
    const RmsPlan p = rms_plan(C / VEC, VEC > 1, 4, 128);
    auto go = [&](auto kernel) { launch_k(kernel, (rows - 1) / p.rpb + 1, p.threads, 0, s, (const T *)x, (int8_t *)q, scale, rows, C, pitch, p.tpr); };
    switch (p.iter) {
    case 1: go(act8_pack_kernel<T, VEC, 1>); break;
    case 2: go(act8_pack_kernel<T, VEC, 2>); break;
    case 4: go(act8_pack_kernel<T, VEC, 4>); break;
    case 8: if (VEC == 1) { go(act8_pack_kernel<T, 1, 8>); break; } return -1;
    case 16: if (VEC == 1) { go(act8_pack_kernel<T, 1, 16>); break; } return -1;
    default: return -1;
    }
    return 1;
}

template <typename T> int pack_wide(const void *x, void *q, float *scale, int rows, int C, const Launch &s) {
    launch_k(act8_pack_wide_kernel<T>, rows, 1024, 0, s, (const T *)x, (int8_t *)q, scale, C, act8_pitch(C));
    return 1;
}

template <typename T> int unpack_as(const void *q, const float *scale, void *x, int rows, int C, const Launch &s) {
    const int pitch = act8_pitch(C);
    const size_t units = (size_t)rows * (pitch / 16);
    const int grid = (int)std::min<size_t>((units + 255) / 256, 148 * 16), vec = C % Vec16<T>::N == 0 && vec_ok(x);
    launch_k(act8_unpack_kernel<T>, grid, 256, 0, s, (const int8_t *)q, scale, (T *)x, units, C, pitch, vec);
    return 1;
}

}  // namespace

int launch_act8_pack(int prec, const void *x, void *q, float *scale, int rows, int C, Launch s) {
    const bool vec = vec_ok(x) && C % (prec == P_BF16 ? 8 : 4) == 0;
    if (C > kRmsMaxC) return prec == P_BF16 ? pack_wide<bf16>(x, q, scale, rows, C, s) : pack_wide<float>(x, q, scale, rows, C, s);
    if (prec == P_BF16) return vec ? pack_as<bf16, 8>(x, q, scale, rows, C, s) : pack_as<bf16, 1>(x, q, scale, rows, C, s);
    return vec ? pack_as<float, 4>(x, q, scale, rows, C, s) : pack_as<float, 1>(x, q, scale, rows, C, s);
}

int launch_act8_unpack(int prec, const void *q, const float *scale, void *x, int rows, int C, Launch s) {
    return prec == P_BF16 ? unpack_as<bf16>(q, scale, x, rows, C, s) : unpack_as<float>(q, scale, x, rows, C, s);
}

}  // namespace ddg

// Activation checkpoints in 8 bits: rows of a tensor to codes with a scale per row, and back (act8.cuh has the formulas).
//
// Bound by memory: packing reads a row once and writes half (bf16) or a quarter (fp32) of its bytes, unpacking the reverse.  A row
// stays on the chip between its maximum and its codes: in shared memory where there are many rows (row_ring.cuh), in its threads'
// registers where there are few or narrow ones; rows of more than 16384 values are read twice.  Measured: 8192 x 4096 bf16 packed
// in 20.8 us (4.8 TB/s; a block per row without copies ahead took 47 us), unpacked in 17.2 us (5.8 TB/s); 8192 x 1021, whose rows
// keep to no boundary, 15 and 8 us; 8192 x 8192 fp32 70 and 55 us (4.8 and 6.1 TB/s); 2048 x 65536 bf16 170 and 67 us.
#include <algorithm>

#include "act8.cuh"
#include "common.cuh"
#include "lm_ops.h"
#include "row_io.cuh"
#include "row_ring.cuh"

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
            act8_store<sizeof(T) == 2 ? kBf16 : kF32, VEC>(to + c, v[i], r);
        }
    }
    for (int c = C + t; c < pitch; c += tpr) to[c] = 0;
}

// The same for many rows: resident blocks walk stretches of them, the rows ahead on their way through shared memory.
template <typename T, int VEC, int ITER>
__global__ void __launch_bounds__(512, 1) act8_pack_ring_kernel(const T *__restrict__ x, int8_t *__restrict__ q, float *__restrict__ scale, int rows, int C, int pitch,
                                                                const __grid_constant__ RingShape shape) {
    constexpr int P = VEC * ITER / 2, G = kGroup<VEC>;  // pairs of a thread, of a group
    extern __shared__ __align__(16) uint8_t ring_smem[];
    __shared__ uint64_t full[kRingMostStages];
    __shared__ __align__(16) float red[6][32];
    __shared__ int flags[2];
    const int t = threadIdx.x, threads = blockDim.x;
    __shared__ const uint8_t *list[1];
    RowRing<1> ring(shape, smem_u32(ring_smem), full, flags, list, {x});
    if (t == 0) ring.init();
    if (t < 32) {
#pragma unroll
        for (int k = 0; k < 6; ++k) red[k][t] = 0.f;
    }
    __syncthreads();
    pdl_launch();
    pdl_wait();
    const int first = (int)((long)rows * blockIdx.x / gridDim.x), last = (int)((long)rows * (blockIdx.x + 1) / gridDim.x);
    for (int row = first; row < min(first + shape.stages, last); ++row) ring.copy(row, -1);
    uint32_t round = 0;
    for (int row = first; row < last; ++row) {
        const bool ok = ring.wait<T, VEC>(row);
        const uint32_t slot = ring.slot(0);
        const int phase = ring_phase(shape, row);
        ring.next();
        F2 v[P];
        uint32_t top = ok ? 0u : 0x7fffffffu;  // a row that did not come is NaN
#pragma unroll
        for (int i = 0; i < P / G; ++i) {
            F2 in[G];
            slot_load<T, VEC>(slot, phase, C, threads, i, in);
#pragma unroll
            for (int j = 0; j < G; ++j) {
                v[i * G + j] = in[j];
                const float2 p = parts(in[j]);
                top = max(top, max(magnitude_bits(p.x), magnitude_bits(p.y)));
            }
        }
        top = ring_max(top, threads >> 5, red, round);
        if (row > first && row - 1 + shape.stages < last) ring.copy(row - 1 + shape.stages, row);
        float s;
        const Act8Row r = act8_row(top, s);
        if (t == 0) scale[row] = s;
        int8_t *to = q + (size_t)row * pitch;
        act8_share_store<sizeof(T) == 2 ? kBf16 : kF32, VEC, ITER>(to, C, threads, v, r);
        for (int c = C + t; c < pitch; c += threads) to[c] = 0;
    }
    if (t == 0) ring.drain();
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

// 16 codes of a row at a time, four of them on their way per thread.
template <typename T>
__global__ void __launch_bounds__(256) act8_unpack_kernel(const int8_t *__restrict__ q, const float *__restrict__ scale, T *__restrict__ x, size_t units, int C, int pitch, int whole) {
    constexpr int kAhead = 4;
    pdl_launch();
    pdl_wait();
    const unsigned per_row = pitch / 16;
    for (size_t i0 = (size_t)blockIdx.x * (256 * kAhead) + threadIdx.x; i0 < units; i0 += (size_t)gridDim.x * (256 * kAhead)) {
        uint4 w[kAhead];
        float s[kAhead];
        size_t row[kAhead];
        int col[kAhead];
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            const size_t i = min(i0 + 256 * u, units - 1);
            row[u] = units <= 0xffffffffu ? (unsigned)i / per_row : i / per_row;
            col[u] = (int)(i - row[u] * per_row) * 16;
            w[u] = *reinterpret_cast<const uint4 *>(q + row[u] * pitch + col[u]);
            s[u] = scale[row[u]];
        }
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            if (i0 + 256 * u >= units) break;
            const uint32_t word[4] = {w[u].x, w[u].y, w[u].z, w[u].w};
            const int c = col[u];
            T *to = x + row[u] * C + c;
            float v[16];
#pragma unroll
            for (int j = 0; j < 16; ++j) v[j] = (float)(int8_t)(word[j / 4] >> (8 * (j % 4))) * s[u];
            constexpr int N = Vec16<T>::N;
            if (whole) {  // 32-byte sectors
#pragma unroll
                for (int j = 0; j < 16; j += 2 * N) {
                    uint32_t o[8];
#pragma unroll
                    for (int k = 0; k < 8; ++k) o[k] = sizeof(T) == 2 ? pack2(v[sizeof(T) == 2 ? 2 * k : 0], v[sizeof(T) == 2 ? 2 * k + 1 : 0]) : __float_as_uint(v[(j + k) % 16]);
                    st_global_32(to + j, o);
                }
            } else {
#pragma unroll
                for (int j = 0; j < 16; j += N)
                    if (c + j < C) store_f<T, N>(to + j, reinterpret_cast<const float(&)[N]>(v[j]));
            }
        }
    }
}

// Rows that keep to no boundary: 256 codes of a row per warp at a time, neighbouring ones to neighbouring lanes.
template <typename T>
__global__ void __launch_bounds__(256) act8_unpack_any_kernel(const int8_t *__restrict__ q, const float *__restrict__ scale, T *__restrict__ x, size_t units, int C, int pitch) {
    constexpr int kCols = 256;
    pdl_launch();
    pdl_wait();
    const unsigned per_row = (C + kCols - 1) / kCols;
    const int lane = threadIdx.x & 31;
    for (size_t i = (size_t)blockIdx.x * 8 + (threadIdx.x >> 5); i < units; i += (size_t)gridDim.x * 8) {
        const size_t row = units <= 0xffffffffu ? (unsigned)i / per_row : i / per_row;
        const int c0 = (int)(i - row * per_row) * kCols + lane;
        const int8_t *from = q + row * pitch;
        const float s = scale[row];
        int8_t v[kCols / 32];
#pragma unroll
        for (int k = 0; k < kCols / 32; ++k)
            if (c0 + 32 * k < C) v[k] = from[c0 + 32 * k];
#pragma unroll
        for (int k = 0; k < kCols / 32; ++k)
            if (c0 + 32 * k < C) x[row * C + c0 + 32 * k] = from_f<T>((float)v[k] * s);
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

template <typename T, int VEC, int ITER> int pack_ring(const void *x, void *q, float *scale, int rows, int C, const RingPlan &p, const Launch &s) {
    static thread_local int ready = -1;
    if (!ring_ready(act8_pack_ring_kernel<T, VEC, ITER>, ready)) return -1;
    launch_k(act8_pack_ring_kernel<T, VEC, ITER>, std::min(rows, 148 * p.per_sm), p.threads, p.smem, s, (const T *)x, (int8_t *)q, scale, rows, C, act8_pitch(C),
             ring_shape(rows, C * (int)sizeof(T), 1, p.smem, block8_polls()));
    return 1;
}

template <typename T> int pack_wide(const void *x, void *q, float *scale, int rows, int C, const Launch &s) {
    launch_k(act8_pack_wide_kernel<T>, rows, 1024, 0, s, (const T *)x, (int8_t *)q, scale, C, act8_pitch(C));
    return 1;
}

template <typename T> int unpack_as(const void *q, const float *scale, void *x, int rows, int C, const Launch &s) {
    const int pitch = act8_pitch(C);
    if (C % Vec16<T>::N != 0 || !vec_ok(x)) {
        const size_t units = (size_t)rows * ((C + 255) / 256);
        launch_k(act8_unpack_any_kernel<T>, (int)std::min<size_t>((units + 7) / 8, 148 * 16), 256, 0, s, (const int8_t *)q, scale, (T *)x, units, C, pitch);
        return 1;
    }
    const size_t units = (size_t)rows * (pitch / 16);
    const int whole = C % 16 == 0 && (reinterpret_cast<uintptr_t>(x) & 31) == 0;
    launch_k(act8_unpack_kernel<T>, (int)std::min<size_t>((units + 1023) / 1024, 148 * 8), 256, 0, s, (const int8_t *)q, scale, (T *)x, units, C, pitch, whole);
    return 1;
}

}  // namespace

int launch_act8_pack(int prec, const void *x, void *q, float *scale, int rows, int C, Launch s) {
    const bool vec = vec_ok(x) && C % (prec == P_BF16 ? 8 : 4) == 0;
    const int per_vec = vec ? (prec == P_BF16 ? 8 : 4) : 1, iter = vec ? 4 : 8;
    if (rows >= 2 * 148 && vec_ok(x) && ring_threads((C + per_vec - 1) / per_vec, iter) >= 64) {  // narrow rows are a warp's of the other kernel
        const RingPlan p = ring_plan(C, C * (int)elem_size(prec), per_vec, iter, 1, 0, 96);
        if (p.threads) {
            if (prec == P_BF16) return vec ? pack_ring<bf16, 8, 4>(x, q, scale, rows, C, p, s) : pack_ring<bf16, 1, 8>(x, q, scale, rows, C, p, s);
            return vec ? pack_ring<float, 4, 4>(x, q, scale, rows, C, p, s) : pack_ring<float, 1, 8>(x, q, scale, rows, C, p, s);
        }
    }
    if (C > kRmsMaxC) return prec == P_BF16 ? pack_wide<bf16>(x, q, scale, rows, C, s) : pack_wide<float>(x, q, scale, rows, C, s);
    if (prec == P_BF16) return vec ? pack_as<bf16, 8>(x, q, scale, rows, C, s) : pack_as<bf16, 1>(x, q, scale, rows, C, s);
    return vec ? pack_as<float, 4>(x, q, scale, rows, C, s) : pack_as<float, 1>(x, q, scale, rows, C, s);
}

int launch_act8_unpack(int prec, const void *q, const float *scale, void *x, int rows, int C, Launch s) {
    return prec == P_BF16 ? unpack_as<bf16>(q, scale, x, rows, C, s) : unpack_as<float>(q, scale, x, rows, C, s);
}

}  // namespace ddg

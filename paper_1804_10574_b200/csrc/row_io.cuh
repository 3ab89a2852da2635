// Rows that stay in the registers of their threads: reductions over a row, vectors of rows of any width, and the split of
// a row over threads.  Used by the norms and by the 8-bit rows.
#pragma once
#include <algorithm>

#include "common.cuh"

namespace ddg {

namespace {

// Sum (or maximum) over the threads of a row: a warp, or the block through shared memory.  Every thread gets the result.
template <bool MAX> __device__ __forceinline__ float row_reduce(float v, bool one_warp, float *red) {
    v = MAX ? warp_max(v) : warp_sum(v);
    if (one_warp) return v;
    const int nw = blockDim.x >> 5, lane = threadIdx.x & 31;
    __syncthreads();  // the previous reduction's values are read
    if (lane == 0) red[threadIdx.x >> 5] = v;
    __syncthreads();
    v = lane < nw ? red[lane] : (MAX ? -INFINITY : 0.f);
    return MAX ? warp_max(v) : warp_sum(v);
}

// threads that rms_plan gives a row of at most 16384 values
constexpr int rms_max_threads(int vec, int iter) { return (vec == 4 && iter == 4) || (vec == 1 && iter == 16) ? 1024 : 512; }

// A thread's values of a vector to 32-bit memory that starts on a 16-byte boundary (VEC > 1), at most 16 bytes at a time.
template <int VEC> __device__ __forceinline__ void store_share(float *p, const float (&v)[VEC]) {
    constexpr int kPart = VEC < 4 ? VEC : 4;
#pragma unroll
    for (int i = 0; i < VEC; i += kPart) {
        float part[kPart];
#pragma unroll
        for (int j = 0; j < kPart; ++j) part[j] = v[i + j];
        store_f<float, kPart>(p + i, part);
    }
}

// Rows of an odd width start anywhere.  SHIFT: a row's vectors are those of the tensor, aligned ones, so that its first and
// last may be shared with its neighbours: vector i has the columns i VEC - phase .. + VEC - 1, phase = row C mod VEC, and of
// a shared one the row's own columns are read and written singly, the others are zeros.  gamma, which starts at column
// zero, is read singly.  Against rows read a value at a time, 1264 x 2933: bf16 forward 10.9 -> 8.0 us, to e4m3 16.6 -> 9.5 us,
// backward 25 -> 21 us; fp32 9.9 -> 8.5, 15.6 -> 10.1 and 25 -> 14 us.
__device__ __forceinline__ bool rms_whole(int c, int vec, int C) { return c >= 0 && c + vec <= C; }
template <typename T, int VEC, bool SHIFT> __device__ __forceinline__ void rms_load(const T *p, int c, int C, float (&v)[VEC]) {
    if (!SHIFT || rms_whole(c, VEC, C)) {
        load_f<T, VEC>(p + c, v);
    } else {
#pragma unroll
        for (int j = 0; j < VEC; ++j) v[j] = c + j >= 0 && c + j < C ? to_f(p[c + j]) : 0.f;
    }
}
template <typename T, int VEC, bool SHIFT> __device__ __forceinline__ void rms_store(T *p, int c, int C, const float (&v)[VEC]) {
    if (!SHIFT || rms_whole(c, VEC, C)) {
        store_f<T, VEC>(p + c, v);
    } else {
#pragma unroll
        for (int j = 0; j < VEC; ++j)
            if (c + j >= 0 && c + j < C) p[c + j] = from_f<T>(v[j]);
    }
}
template <typename T, int VEC, bool SHIFT> __device__ __forceinline__ void rms_gamma(const T *__restrict__ gamma, int c, int C, float (&v)[VEC]) {
    if (!SHIFT) {
        load_f<T, VEC>(gamma + c, v);
    } else {
#pragma unroll
        for (int j = 0; j < VEC; ++j) v[j] = c + j >= 0 && c + j < C ? to_f(gamma[c + j]) : 0.f;
    }
}

// One row's share of a thread as it lies in memory.
template <typename T, int VEC, int ITER, bool SHIFT> struct RawRow {
    Pack<T, VEC> v[ITER];
    __device__ __forceinline__ void load1(int i, const T *p, int c, int C, bool single = false) {
        if (!SHIFT || (!single && rms_whole(c, VEC, C))) {
            v[i] = *reinterpret_cast<const Pack<T, VEC> *>(p + c);
        } else {
#pragma unroll
            for (int j = 0; j < VEC; ++j) v[i].v[j] = c + j >= 0 && c + j < C ? p[c + j] : from_f<T>(0.f);
        }
    }
    __device__ __forceinline__ void load(const T *p, int t, int tpr, int C, int phase, bool single = false) {
#pragma unroll
        for (int i = 0; i < ITER; ++i) {
            const int c = (i * tpr + t) * VEC - phase;
            if (c < C) load1(i, p, c, C, single);
        }
    }
    __device__ __forceinline__ float at(int i, int j) const { return to_f(v[i].v[j]); }
};

// ---- host side ---------------------------------------------------------------------------------------------------
inline bool vec_ok(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }

// threads of a row, vectors per thread, threads of a block and rows of a block
struct RmsPlan { int tpr, iter, threads, rpb; };
inline RmsPlan rms_plan(int nvec, bool vec, int warp_iters, int warp_threads) {
    RmsPlan p;
    const int warp_iter = (nvec + 31) / 32;
    if (warp_iter <= warp_iters) {
        p.iter = warp_iter <= 1 ? 1 : (warp_iter <= 2 ? 2 : 4);
        p.tpr = 32; p.threads = warp_threads; p.rpb = warp_threads / 32;
        return p;
    }
    p.iter = 1;
    while (p.iter < (vec ? 4 : 16) && nvec > p.iter * 512) p.iter *= 2;
    p.threads = std::min(1024, ((nvec + p.iter - 1) / p.iter + 31) / 32 * 32);
    p.tpr = p.threads; p.rpb = 1;
    return p;
}
// Vectors of a row: with SHIFT the most that a phase can take.  Rows that would need more threads than a kernel has are read
// a value at a time.
inline int rms_nvec(int C, int vec, bool shift) { return shift ? (C + 2 * vec - 2) / vec : C / vec; }
inline bool rms_shift_fits(int C, int vec) { return rms_nvec(C, vec, true) <= (vec == 8 ? 2048 : 4096); }

}  // namespace

}  // namespace ddg

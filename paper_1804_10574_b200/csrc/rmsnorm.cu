// Root-mean-square norm with the residual's addition, its 8-bit output and its backward pass.
//
//   h = x + res;  r = 1 / sqrt(mean(h^2) + eps);  y = h r gamma;  q = e4m3(y / s), s = amax(|y| of the group) / 448
//   dx = dh + r (gamma dy - h r^2 mean(gamma dy h));  dgamma = sum over rows of dy h r
//
// Bound by memory: the forward pass reads x and res and writes h and y (or q) once, the backward pass reads dy, h and dh
// and writes dx once.  A row stays in the registers of its threads between the loads, the reduction and the stores; y is
// taken from the unrounded sum.  A row of at most four 16-byte vectors per lane is one warp's (no barrier), a longer one a
// block's.  Measured at 8192 x 4096 bf16: forward 42 us (6.4 TB/s), to e4m3 46 us (5.1 TB/s, more than a third of it
// instructions), backward 51 us with the fold of dgamma (5.3 TB/s).
#include <cuda_fp8.h>
#include <float.h>

#include <algorithm>

#include "cluster.cuh"
#include "common.cuh"
#include "lm_ops.h"

namespace ddg {

namespace {

constexpr float kE4m3Max = 448.f;

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

// what rms_plan gives a row of at most 16384 values
constexpr int kRmsCluster = 8;
constexpr int kWarpRowThreads = 256;  // of a backward block whose warps have a row each
constexpr int rms_max_threads(int vec, int iter) { return (vec == 4 && iter == 4) || (vec == 1 && iter == 16) ? 1024 : 512; }

template <int VEC> __device__ __forceinline__ void store_q(uint8_t *p, const float (&v)[VEC]) {
    if (VEC == 1) {
        *p = __nv_cvt_float_to_fp8(v[0], __NV_SATFINITE, __NV_E4M3);
    } else {
        uint16_t w[(VEC + 1) / 2];
#pragma unroll
        for (int j = 0; j < VEC / 2; ++j) w[j] = __nv_cvt_float2_to_fp8x2(make_float2(v[2 * j], v[2 * j + 1]), __NV_SATFINITE, __NV_E4M3);
        if (VEC == 8)
            *reinterpret_cast<uint2 *>(p) = make_uint2((uint32_t)w[0] | ((uint32_t)w[1] << 16), (uint32_t)w[VEC == 8 ? 2 : 0] | ((uint32_t)w[VEC == 8 ? 3 : 0] << 16));
        else
            *reinterpret_cast<uint32_t *>(p) = (uint32_t)w[0] | ((uint32_t)w[1] << 16);
    }
}

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

// x, res, h and y may be the same tensor (a thread reads its elements before it writes them).  group: 128 (vector forms
// only: 128 / VEC neighbouring lanes hold a group) or 0 (the row).
// Registers for four blocks of 512 threads per SM: with three, 4096 x 8192 took 44.3 us instead of 42.1.
template <typename T, int VEC, int ITER, bool SHIFT>
__global__ void __launch_bounds__(rms_max_threads(VEC, ITER), ITER <= 2 ? 4 : (VEC == 8 ? 2 : 1)) rms_fwd_kernel(const T *x, const T *res, const T *__restrict__ gamma, T *h, T *y, uint8_t *__restrict__ q,
                                                       float *__restrict__ scale, float *__restrict__ rstd, int rows, int C, int tpr, int group, float eps) {
    __shared__ float red[32];
    pdl_launch();
    pdl_wait();
    const bool one_warp = tpr == 32;
    const int t = one_warp ? (threadIdx.x & 31) : threadIdx.x;
    const int row = one_warp ? blockIdx.x * (blockDim.x >> 5) + (threadIdx.x >> 5) : blockIdx.x;
    if (row >= rows) return;  // whole warps, and only where a row is one warp's
    const size_t at = (size_t)row * C;
    const int phase = SHIFT ? (int)(at % VEC) : 0;
    float v[ITER][VEC];
    float ss = 0.f;
#pragma unroll
    for (int i = 0; i < ITER; ++i) {
        const int c = (i * tpr + t) * VEC - phase;
        if (c < C) {
            rms_load<T, VEC, SHIFT>(x + at, c, C, v[i]);
            if (res) {
                float b[VEC];
                rms_load<T, VEC, SHIFT>(res + at, c, C, b);
#pragma unroll
                for (int j = 0; j < VEC; ++j) v[i][j] += b[j];
            }
        } else {
#pragma unroll
            for (int j = 0; j < VEC; ++j) v[i][j] = 0.f;
        }
    }
#pragma unroll
    for (int i = 0; i < ITER; ++i) {
        const int c = (i * tpr + t) * VEC - phase;
        if (h && c < C) rms_store<T, VEC, SHIFT>(h + at, c, C, v[i]);
#pragma unroll
        for (int j = 0; j < VEC; ++j) ss = fmaf(v[i][j], v[i][j], ss);
    }
    ss = row_reduce<false>(ss, one_warp, red);
    const float r = rsqrtf(ss / (float)C + eps);
    if (rstd && t == 0) rstd[row] = r;
#pragma unroll
    for (int i = 0; i < ITER; ++i) {
        const int c = (i * tpr + t) * VEC - phase;
        if (c < C) {
            float g[VEC];
            rms_gamma<T, VEC, SHIFT>(gamma, c, C, g);
#pragma unroll
            for (int j = 0; j < VEC; ++j) v[i][j] = v[i][j] * r * g[j];
            if (y) rms_store<T, VEC, SHIFT>(y + at, c, C, v[i]);
        }
    }
    if (!q) return;
    float top[ITER];
    float all = 0.f;
#pragma unroll
    for (int i = 0; i < ITER; ++i) {
        top[i] = 0.f;
#pragma unroll
        for (int j = 0; j < VEC; ++j) top[i] = fmaxf(top[i], fabsf(v[i][j]));
        all = fmaxf(all, top[i]);
    }
    if (group == 0) {
        all = row_reduce<true>(all, one_warp, red);
    } else {
#pragma unroll
        for (int i = 0; i < ITER; ++i)
#pragma unroll
            for (int o = 64 / VEC; o > 0; o >>= 1)
                if (o < 32) top[i] = fmaxf(top[i], __shfl_xor_sync(0xffffffffu, top[i], o));
    }
#pragma unroll
    for (int i = 0; i < ITER; ++i) {
        const int c = (i * tpr + t) * VEC - phase;
        if (c < C) {
            const float a = group == 0 ? all : top[i];
            // a group of zeros (or of NaN) has scale 1; 1 / s stays finite
            const float s = a > 0.f ? fmaxf(a / kE4m3Max, FLT_MIN) : 1.f;
            const float inv = 1.f / s, finite = fminf(s, FLT_MAX);
            // v / s: the product with the reciprocal may be a unit of fp32 off, which at a border of e4m3 is a whole step.  One
            // correction by the remainder (Markstein, 1990) takes that away; 4096 x 8192 bf16 44.0 -> 45.8 us, 51.3 with divisions.
#pragma unroll
            for (int j = 0; j < VEC; ++j) {
                const float t = v[i][j] * inv;
                v[i][j] = fmaf(fmaf(-t, finite, v[i][j]), inv, t);
            }
            if (!SHIFT || rms_whole(c, VEC, C)) {
                store_q<VEC>(q + at + c, v[i]);
            } else {
#pragma unroll
                for (int j = 0; j < VEC; ++j)
                    if (c + j >= 0 && c + j < C) q[at + c + j] = __nv_cvt_float_to_fp8(v[i][j], __NV_SATFINITE, __NV_E4M3);
            }
            if (group == 0) { if (t == 0 && i == 0) scale[row] = s; }
            else if (c % 128 == 0) scale[(size_t)row * (C / 128) + c / 128] = s;
        }
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

// Blocks (or warps, where a row is one warp's) walk the rows; each keeps its share of dgamma in registers, a block's warps
// add theirs up, and part[block][C] goes to the folding kernel.  With up to two vectors a thread, the next row's dy, h and dh
// are loaded before this row's reduction, so that memory stays busy through its two barriers; with more there are no
// registers for it.  Few rows are one cluster's (dgamma given), whose blocks fold their shares over one another's shared
// memory instead: one launch less, which is what such a call costs.  dx may be dy, dh or h: a row is written after it was read, and the row that is loaded ahead is
// the same walker's.
template <typename T, int VEC, int ITER, bool WARP, bool SHIFT>
__global__ void __launch_bounds__(WARP ? kWarpRowThreads : rms_max_threads(VEC, ITER), WARP ? (ITER == 1 ? 3 : 2) : (ITER == 1 ? 2 : 1))
rms_bwd_kernel(const T *dy, const T *dh, const T *h, const T *__restrict__ gamma, const float *__restrict__ rstd, T *dx, float *__restrict__ part, int rows, int C,
               float *__restrict__ dgamma) {
    constexpr bool kAhead = ITER <= 2;
    __shared__ float red[32];
    extern __shared__ float shares[];  // WARP: [warps][C]; then, in a cluster, the block's [C]
    pdl_launch();
    pdl_wait();
    const int warp = threadIdx.x >> 5, warps = blockDim.x >> 5;
    const int tpr = WARP ? 32 : blockDim.x, t = WARP ? (threadIdx.x & 31) : threadIdx.x;
    const int walkers = WARP ? gridDim.x * warps : gridDim.x;
    int row = WARP ? blockIdx.x * warps + warp : blockIdx.x;
    const int phase = SHIFT ? (int)((size_t)row * C % VEC) : 0;  // of all the walker's rows: with SHIFT walkers is a multiple of VEC, or there is one row each
    float acc[ITER][VEC];
#pragma unroll
    for (int i = 0; i < ITER; ++i)
#pragma unroll
        for (int j = 0; j < VEC; ++j) acc[i][j] = 0.f;
    typedef RawRow<T, VEC, ITER, SHIFT> Raw;
    Raw g, a, b, d, next_a, next_b, next_d;
    float r = 0.f, next_r = 0.f;
    if (kAhead) g.load(gamma, t, tpr, C, phase, true);
    if (row < rows) {
        a.load(dy + (size_t)row * C, t, tpr, C, phase);
        b.load(h + (size_t)row * C, t, tpr, C, phase);
        if (dh && kAhead) d.load(dh + (size_t)row * C, t, tpr, C, phase);
        r = rstd[row];
    }
    for (; row < rows; row += walkers) {
        if (kAhead && row + walkers < rows) {
            const size_t next = (size_t)(row + walkers) * C;
            next_a.load(dy + next, t, tpr, C, phase);
            next_b.load(h + next, t, tpr, C, phase);
            if (dh) next_d.load(dh + next, t, tpr, C, phase);
            next_r = rstd[row + walkers];
        }
        float dot = 0.f;
#pragma unroll
        for (int i = 0; i < ITER; ++i) {
            const int c = (i * tpr + t) * VEC - phase;
            if (c < C) {
                float w[VEC];
                if (!kAhead) rms_gamma<T, VEC, SHIFT>(gamma, c, C, w);
#pragma unroll
                for (int j = 0; j < VEC; ++j) {
                    const float y = a.at(i, j), x = b.at(i, j);
                    acc[i][j] = fmaf(y, x * r, acc[i][j]);
                    dot = fmaf(y * (kAhead ? g.at(i, j) : w[j]), x, dot);
                }
            }
        }
        dot = row_reduce<false>(dot, WARP, red);
        const float k = dot / (float)C * r * r;
#pragma unroll
        for (int i = 0; i < ITER; ++i) {
            const int c = (i * tpr + t) * VEC - phase;
            if (c < C) {
                float w[VEC], o[VEC];
                if (!kAhead) {
                    rms_gamma<T, VEC, SHIFT>(gamma, c, C, w);
                    if (dh) d.load1(i, dh + (size_t)row * C, c, C);
                }
#pragma unroll
                for (int j = 0; j < VEC; ++j) o[j] = fmaf(r, a.at(i, j) * (kAhead ? g.at(i, j) : w[j]) - b.at(i, j) * k, dh ? d.at(i, j) : 0.f);
                rms_store<T, VEC, SHIFT>(dx + (size_t)row * C, c, C, o);
            }
        }
        if (kAhead) {
            a = next_a; b = next_b; d = next_d; r = next_r;
        } else if (row + walkers < rows) {
            a.load(dy + (size_t)(row + walkers) * C, t, tpr, C, phase);
            b.load(h + (size_t)(row + walkers) * C, t, tpr, C, phase);
            r = rstd[row + walkers];
        }
    }
    float *own = dgamma ? shares + (WARP ? warps * ((C + 3) & ~3) : 0) : part + (size_t)blockIdx.x * C;
#pragma unroll
    for (int i = 0; i < ITER; ++i) {
        const int c = (i * tpr + t) * VEC - phase;
        float *to = WARP ? shares + warp * ((C + 3) & ~3) : own;
        if (SHIFT) {
#pragma unroll
            for (int j = 0; j < VEC; ++j)
                if (c + j >= 0 && c + j < C) to[c + j] = acc[i][j];
        } else if (c < C) {
            store_share<VEC>(to + c, acc[i]);
        }
    }
    if (WARP) {
        __syncthreads();
        for (int c = threadIdx.x; c < C; c += blockDim.x) {
            float sum = shares[c];
            for (int w = 1; w < warps; ++w) sum += shares[w * ((C + 3) & ~3) + c];
            own[c] = sum;
        }
    }
    if (dgamma) {  // a block's slice of the columns, blocks in index order
        __syncthreads();
        cluster_sync();
        const uint32_t base = (uint32_t)__cvta_generic_to_shared(own);
        for (int c = (int)cluster_rank() * blockDim.x + threadIdx.x; c < C; c += kRmsCluster * blockDim.x) {
            float sum = 0.f;
#pragma unroll
            for (int r = 0; r < kRmsCluster; ++r) {
                float v;
                asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(map_rank(base + 4u * c, r)));
                sum += v;
            }
            dgamma[c] = sum;
        }
        cluster_sync();  // no block leaves while its share is read
    }
}

// dgamma[c] = sum over walkers, 32 columns per block, walkers in index order per warp and warps in index order
__global__ void __launch_bounds__(1024) rms_fold_kernel(const float *__restrict__ part, int walkers, float *__restrict__ dgamma, int C) {
    __shared__ float fold[32][32];
    pdl_launch();
    pdl_wait();
    const int lane = threadIdx.x & 31, w = threadIdx.x >> 5, c = blockIdx.x * 32 + lane;
    float a = 0.f;
    if (c < C) {
#pragma unroll 8
        for (int i = w; i < walkers; i += 32) a += part[(size_t)i * C + c];
    }
    fold[w][lane] = a;
    __syncthreads();
    if (w == 0 && c < C) {
        for (int i = 1; i < 32; ++i) a += fold[i][lane];
        dgamma[c] = a;
    }
}

bool vec_ok(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }

// threads of a row, vectors per thread, threads of a block and rows of a block
struct RmsPlan { int tpr, iter, threads, rpb; };
RmsPlan rms_plan(int nvec, bool vec, int warp_iters, int warp_threads) {
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
RmsPlan rms_fwd_plan(int nvec, bool vec) { return rms_plan(nvec, vec, 4, 128); }
RmsPlan rms_bwd_plan(int nvec, bool vec) { return rms_plan(nvec, vec, 2, kWarpRowThreads); }
// Vectors of a row: with SHIFT the most that a phase can take.  Rows that would need more threads than a kernel has are read
// a value at a time.
int rms_nvec(int C, int vec, bool shift) { return shift ? (C + 2 * vec - 2) / vec : C / vec; }
bool rms_shift_fits(int C, int vec) { return rms_nvec(C, vec, true) <= (vec == 8 ? 2048 : 4096); }
// Blocks of the backward pass: as many as the kernel's registers (its launch bounds) let stay resident, so that none waits
// for a second round with rows of its own; with SHIFT a multiple of eight where there are rows for it.
int rms_bwd_blocks(const RmsPlan &p, int rows, bool shift) {
    const int per_sm = p.tpr == 32 ? (p.iter == 1 ? 3 : 2) : std::max(1, (p.iter == 1 ? 1024 : 512) / p.threads);
    return std::min((rows + p.rpb - 1) / p.rpb, shift ? 148 * per_sm / 8 * 8 : 148 * per_sm);
}

}  // namespace

size_t rmsnorm_scratch_elems(int rows, int C) {
    int most = rms_bwd_blocks(rms_bwd_plan(C, false), rows, false);
    for (int vec : {4, 8})
        if (C % vec == 0 || rms_shift_fits(C, vec)) most = std::max(most, rms_bwd_blocks(rms_bwd_plan(rms_nvec(C, vec, C % vec != 0), true), rows, C % vec != 0));
    return (size_t)most * C;
}

template <typename T, int VEC, bool SHIFT = false>
static int rms_fwd(const void *x, const void *res, const void *gamma, void *h, void *y, void *y8, float *scale8, float *rstd, int rows, int C, int group,
                   float eps, const Launch &s) {
    const RmsPlan p = rms_fwd_plan(rms_nvec(C, VEC, SHIFT), VEC > 1);
    const int grid = (rows - 1) / p.rpb + 1;
    auto go = [&](auto kernel) {
        launch_k(kernel, grid, p.threads, 0, s, (const T *)x, (const T *)res, (const T *)gamma, (T *)h, (T *)y, (uint8_t *)y8, scale8, rstd, rows, C, p.tpr, group, eps);
    };
    switch (p.iter) {
    case 1: go(rms_fwd_kernel<T, VEC, 1, SHIFT>); break;
    case 2: go(rms_fwd_kernel<T, VEC, 2, SHIFT>); break;
    case 4: go(rms_fwd_kernel<T, VEC, 4, SHIFT>); break;
    case 8: if (VEC == 1) { go(rms_fwd_kernel<T, 1, 8, false>); break; } return -1;
    case 16: if (VEC == 1) { go(rms_fwd_kernel<T, 1, 16, false>); break; } return -1;
    default: return -1;
    }
    return 1;
}

template <typename T, int VEC, bool SHIFT = false>
static int rms_bwd(const void *dy, const void *dh, const void *h, const void *gamma, const float *rstd, void *dx, float *dgamma, float *scratch, int rows, int C,
                   const Launch &s) {
    const RmsPlan p = rms_bwd_plan(rms_nvec(C, VEC, SHIFT), VEC > 1);
    // one cluster of eight blocks while a warp (or block) has at most four rows
    const bool cluster = rows <= kRmsCluster * p.rpb * 4 && (p.tpr == 32 || C <= 8192);
    const int grid = cluster ? kRmsCluster : rms_bwd_blocks(p, rows, SHIFT);
    auto go = [&](auto kernel, size_t smem) {
        cudaLaunchConfig_t cfg = {};
        cfg.gridDim = dim3(grid); cfg.blockDim = dim3(p.threads); cfg.stream = s.s;
        cfg.dynamicSmemBytes = smem + (cluster ? (size_t)C * sizeof(float) : 0);
        cudaLaunchAttribute attr[2];
        cfg.attrs = attr;
        if (cluster) {
            attr[cfg.numAttrs].id = cudaLaunchAttributeClusterDimension;
            attr[cfg.numAttrs].val.clusterDim.x = kRmsCluster;
            attr[cfg.numAttrs].val.clusterDim.y = attr[cfg.numAttrs].val.clusterDim.z = 1;
            ++cfg.numAttrs;
        }
        if (s.pdl == 1) {
            attr[cfg.numAttrs].id = cudaLaunchAttributeProgrammaticStreamSerialization;
            attr[cfg.numAttrs].val.programmaticStreamSerializationAllowed = 1;
            ++cfg.numAttrs;
        }
        cudaLaunchKernelEx(&cfg, kernel, (const T *)dy, (const T *)dh, (const T *)h, (const T *)gamma, rstd, (T *)dx, scratch, rows, C, cluster ? dgamma : (float *)nullptr);
    };
    if (p.tpr == 32) {
        const size_t smem = (size_t)p.rpb * ((C + 3) & ~3) * sizeof(float);
        if (p.iter == 1) go(rms_bwd_kernel<T, VEC, 1, true, SHIFT>, smem); else go(rms_bwd_kernel<T, VEC, 2, true, SHIFT>, smem);
    } else {
        switch (p.iter) {
        case 1: go(rms_bwd_kernel<T, VEC, 1, false, SHIFT>, 0); break;
        case 2: go(rms_bwd_kernel<T, VEC, 2, false, SHIFT>, 0); break;
        case 4: go(rms_bwd_kernel<T, VEC, 4, false, SHIFT>, 0); break;
        case 8: if (VEC == 1) { go(rms_bwd_kernel<T, 1, 8, false, false>, 0); break; } return -1;
        case 16: if (VEC == 1) { go(rms_bwd_kernel<T, 1, 16, false, false>, 0); break; } return -1;
        default: return -1;
        }
    }
    if (cluster) return 1;
    launch_k(rms_fold_kernel, (C + 31) / 32, 1024, 0, s, (const float *)scratch, grid, dgamma, C);
    return 2;
}

// The vector forms want every tensor on a 16-byte boundary; SHIFT where rows do not keep to it.
int launch_add_rmsnorm_fwd(int prec, const void *x, const void *res, const void *gamma, void *h, void *y, void *y8, float *scale8, float *rstd, int rows, int C,
                           int group, float eps, Launch s) {
    const int vec = prec == P_BF16 ? 8 : 4;
    const bool aligned = vec_ok(x) && vec_ok(res) && vec_ok(gamma) && vec_ok(h) && vec_ok(y) && (reinterpret_cast<uintptr_t>(y8) & 7) == 0;
    const bool v = C % vec == 0 && aligned, shift = C % vec != 0 && aligned && rms_shift_fits(C, vec);
    if (group != 0 && !v) return -1;
    auto go = [&](auto f) { return f(x, res, gamma, h, y, y8, scale8, rstd, rows, C, group, eps, s); };
    if (prec == P_BF16) return v ? go(rms_fwd<bf16, 8>) : (shift ? go(rms_fwd<bf16, 8, true>) : go(rms_fwd<bf16, 1>));
    return v ? go(rms_fwd<float, 4>) : (shift ? go(rms_fwd<float, 4, true>) : go(rms_fwd<float, 1>));
}

int launch_add_rmsnorm_bwd(int prec, const void *dy, const void *dh, const void *h, const void *gamma, const float *rstd, void *dx, float *dgamma, float *scratch,
                           int rows, int C, Launch s) {
    const int vec = prec == P_BF16 ? 8 : 4;
    const bool aligned = vec_ok(dy) && vec_ok(dh) && vec_ok(h) && vec_ok(gamma) && vec_ok(dx) && vec_ok(scratch);
    // Narrow bf16 rows are mostly ends, and each walker reads its gamma singly: a value at a time is faster (4353 x 223: 9.1 us,
    // 12.0 us with SHIFT; 777 x 1021: 7.1 and 9.9 us; fp32 8.8 and 6.8, 6.6 and 6.4 us).
    const bool v = C % vec == 0 && aligned, shift = C % vec != 0 && aligned && rms_shift_fits(C, vec) && (prec == P_F32 || C >= 2048);
    auto go = [&](auto f) { return f(dy, dh, h, gamma, rstd, dx, dgamma, scratch, rows, C, s); };
    if (prec == P_BF16) return v ? go(rms_bwd<bf16, 8>) : (shift ? go(rms_bwd<bf16, 8, true>) : go(rms_bwd<bf16, 1>));
    return v ? go(rms_bwd<float, 4>) : (shift ? go(rms_bwd<float, 4, true>) : go(rms_bwd<float, 1>));
}

}  // namespace ddg

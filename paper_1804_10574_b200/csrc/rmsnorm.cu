// Root-mean-square norm with the residual's addition, its 8-bit output and its backward pass.
//
//   h = x + res;  r = 1 / sqrt(mean(h^2) + eps);  y = h r gamma;  q = e4m3(y / s), s = amax(|y| of the group) / 448
//   dx = dh + r (gamma dy - h r^2 mean(gamma dy h));  dgamma = sum over rows of dy h r
//
// Bound by memory: the forward pass reads x and res and writes h and y (or q) once, the backward pass reads dy, h and dh
// and writes dx once.  A row stays in the registers of its threads between the loads, the reduction and the stores; y is
// taken from the unrounded sum.  A row of at most four 16-byte vectors per lane is one warp's (no barrier), a longer one a
// block's.  Measured at 8192 x 4096 bf16: forward 42 us (6.4 TB/s), to e4m3 44 us (5.4 TB/s, more than a third of it
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

// x, res, h and y may be the same tensor (a thread reads its elements before it writes them).  group: 128 (vector forms
// only: 128 / VEC neighbouring lanes hold a group) or 0 (the row).
// Registers for four blocks of 512 threads per SM: with three, 4096 x 8192 took 44.3 us instead of 42.1.
template <typename T, int VEC, int ITER>
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
    float v[ITER][VEC];
    float ss = 0.f;
#pragma unroll
    for (int i = 0; i < ITER; ++i) {
        const int c = (i * tpr + t) * VEC;
        if (c < C) {
            load_f<T, VEC>(x + at + c, v[i]);
            if (res) {
                float b[VEC];
                load_f<T, VEC>(res + at + c, b);
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
        const int c = (i * tpr + t) * VEC;
        if (h && c < C) store_f<T, VEC>(h + at + c, v[i]);
#pragma unroll
        for (int j = 0; j < VEC; ++j) ss = fmaf(v[i][j], v[i][j], ss);
    }
    ss = row_reduce<false>(ss, one_warp, red);
    const float r = rsqrtf(ss / (float)C + eps);
    if (rstd && t == 0) rstd[row] = r;
#pragma unroll
    for (int i = 0; i < ITER; ++i) {
        const int c = (i * tpr + t) * VEC;
        if (c < C) {
            float g[VEC];
            load_f<T, VEC>(gamma + c, g);
#pragma unroll
            for (int j = 0; j < VEC; ++j) v[i][j] = v[i][j] * r * g[j];
            if (y) store_f<T, VEC>(y + at + c, v[i]);
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
        const int c = (i * tpr + t) * VEC;
        if (c < C) {
            const float a = group == 0 ? all : top[i];
            // a group of zeros (or of NaN) has scale 1; 1 / s stays finite
            const float s = a > 0.f ? fmaxf(a / kE4m3Max, FLT_MIN) : 1.f;
            const float inv = 1.f / s;
#pragma unroll
            for (int j = 0; j < VEC; ++j) v[i][j] *= inv;
            store_q<VEC>(q + at + c, v[i]);
            if (group == 0) { if (t == 0 && i == 0) scale[row] = s; }
            else if (c % 128 == 0) scale[(size_t)row * (C / 128) + c / 128] = s;
        }
    }
}

// One row's share of a thread as it lies in memory.
template <typename T, int VEC, int ITER> struct RawRow {
    Pack<T, VEC> v[ITER];
    __device__ __forceinline__ void load(const T *p, int t, int tpr, int C) {
#pragma unroll
        for (int i = 0; i < ITER; ++i) {
            const int c = (i * tpr + t) * VEC;
            if (c < C) v[i] = *reinterpret_cast<const Pack<T, VEC> *>(p + c);
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
template <typename T, int VEC, int ITER, bool WARP>
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
    float acc[ITER][VEC];
#pragma unroll
    for (int i = 0; i < ITER; ++i)
#pragma unroll
        for (int j = 0; j < VEC; ++j) acc[i][j] = 0.f;
    typedef RawRow<T, VEC, ITER> Raw;
    Raw g, a, b, d, next_a, next_b, next_d;
    float r = 0.f, next_r = 0.f;
    if (kAhead) g.load(gamma, t, tpr, C);
    if (row < rows) {
        a.load(dy + (size_t)row * C, t, tpr, C);
        b.load(h + (size_t)row * C, t, tpr, C);
        if (dh && kAhead) d.load(dh + (size_t)row * C, t, tpr, C);
        r = rstd[row];
    }
    for (; row < rows; row += walkers) {
        if (kAhead && row + walkers < rows) {
            const size_t next = (size_t)(row + walkers) * C;
            next_a.load(dy + next, t, tpr, C);
            next_b.load(h + next, t, tpr, C);
            if (dh) next_d.load(dh + next, t, tpr, C);
            next_r = rstd[row + walkers];
        }
        float dot = 0.f;
#pragma unroll
        for (int i = 0; i < ITER; ++i) {
            const int c = (i * tpr + t) * VEC;
            if (c < C) {
                float w[VEC];
                if (!kAhead) load_f<T, VEC>(gamma + c, w);
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
            const int c = (i * tpr + t) * VEC;
            if (c < C) {
                float w[VEC], o[VEC];
                if (!kAhead) {
                    load_f<T, VEC>(gamma + c, w);
                    if (dh) d.v[i] = *reinterpret_cast<const Pack<T, VEC> *>(dh + (size_t)row * C + c);
                }
#pragma unroll
                for (int j = 0; j < VEC; ++j) o[j] = fmaf(r, a.at(i, j) * (kAhead ? g.at(i, j) : w[j]) - b.at(i, j) * k, dh ? d.at(i, j) : 0.f);
                store_f<T, VEC>(dx + (size_t)row * C + c, o);
            }
        }
        if (kAhead) {
            a = next_a; b = next_b; d = next_d; r = next_r;
        } else if (row + walkers < rows) {
            a.load(dy + (size_t)(row + walkers) * C, t, tpr, C);
            b.load(h + (size_t)(row + walkers) * C, t, tpr, C);
            r = rstd[row + walkers];
        }
    }
    float *own = dgamma ? shares + (WARP ? warps * ((C + 3) & ~3) : 0) : part + (size_t)blockIdx.x * C;
#pragma unroll
    for (int i = 0; i < ITER; ++i) {
        const int c = (i * tpr + t) * VEC;
        if (c < C) store_share<VEC>(WARP ? shares + warp * ((C + 3) & ~3) + c : own + c, acc[i]);
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
// Blocks of the backward pass: as many as the kernel's registers (its launch bounds) let stay resident, so that none waits
// for a second round with rows of its own.
int rms_bwd_blocks(const RmsPlan &p, int rows) {
    const int per_sm = p.tpr == 32 ? (p.iter == 1 ? 3 : 2) : std::max(1, (p.iter == 1 ? 1024 : 512) / p.threads);
    return std::min((rows + p.rpb - 1) / p.rpb, 148 * per_sm);
}

}  // namespace

size_t rmsnorm_scratch_elems(int rows, int C) {
    int most = rms_bwd_blocks(rms_bwd_plan(C, false), rows);
    for (int vec : {4, 8})
        if (C % vec == 0) most = std::max(most, rms_bwd_blocks(rms_bwd_plan(C / vec, true), rows));
    return (size_t)most * C;
}

template <typename T, int VEC>
static int rms_fwd(const void *x, const void *res, const void *gamma, void *h, void *y, void *y8, float *scale8, float *rstd, int rows, int C, int group,
                   float eps, const Launch &s) {
    const RmsPlan p = rms_fwd_plan(C / VEC, VEC > 1);
    const int grid = (rows - 1) / p.rpb + 1;
    auto go = [&](auto kernel) {
        launch_k(kernel, grid, p.threads, 0, s, (const T *)x, (const T *)res, (const T *)gamma, (T *)h, (T *)y, (uint8_t *)y8, scale8, rstd, rows, C, p.tpr, group, eps);
    };
    switch (p.iter) {
    case 1: go(rms_fwd_kernel<T, VEC, 1>); break;
    case 2: go(rms_fwd_kernel<T, VEC, 2>); break;
    case 4: go(rms_fwd_kernel<T, VEC, 4>); break;
    case 8: if (VEC == 1) { go(rms_fwd_kernel<T, 1, 8>); break; } return -1;
    case 16: if (VEC == 1) { go(rms_fwd_kernel<T, 1, 16>); break; } return -1;
    default: return -1;
    }
    return 1;
}

template <typename T, int VEC>
static int rms_bwd(const void *dy, const void *dh, const void *h, const void *gamma, const float *rstd, void *dx, float *dgamma, float *scratch, int rows, int C,
                   const Launch &s) {
    const RmsPlan p = rms_bwd_plan(C / VEC, VEC > 1);
    // one cluster of eight blocks while a warp (or block) has at most four rows
    const bool cluster = rows <= kRmsCluster * p.rpb * 4 && (p.tpr == 32 || C <= 8192);
    const int grid = cluster ? kRmsCluster : rms_bwd_blocks(p, rows);
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
        if (p.iter == 1) go(rms_bwd_kernel<T, VEC, 1, true>, smem); else go(rms_bwd_kernel<T, VEC, 2, true>, smem);
    } else {
        switch (p.iter) {
        case 1: go(rms_bwd_kernel<T, VEC, 1, false>, 0); break;
        case 2: go(rms_bwd_kernel<T, VEC, 2, false>, 0); break;
        case 4: go(rms_bwd_kernel<T, VEC, 4, false>, 0); break;
        case 8: if (VEC == 1) { go(rms_bwd_kernel<T, 1, 8, false>, 0); break; } return -1;
        case 16: if (VEC == 1) { go(rms_bwd_kernel<T, 1, 16, false>, 0); break; } return -1;
        default: return -1;
        }
    }
    if (cluster) return 1;
    launch_k(rms_fold_kernel, (C + 31) / 32, 1024, 0, s, (const float *)scratch, grid, dgamma, C);
    return 2;
}

int launch_add_rmsnorm_fwd(int prec, const void *x, const void *res, const void *gamma, void *h, void *y, void *y8, float *scale8, float *rstd, int rows, int C,
                           int group, float eps, Launch s) {
    const int vec = prec == P_BF16 ? 8 : 4;
    const bool v = C % vec == 0 && vec_ok(x) && vec_ok(res) && vec_ok(gamma) && vec_ok(h) && vec_ok(y) && (reinterpret_cast<uintptr_t>(y8) & 7) == 0;
    if (group != 0 && !v) return -1;
    if (prec == P_BF16)
        return v ? rms_fwd<bf16, 8>(x, res, gamma, h, y, y8, scale8, rstd, rows, C, group, eps, s) : rms_fwd<bf16, 1>(x, res, gamma, h, y, y8, scale8, rstd, rows, C, group, eps, s);
    return v ? rms_fwd<float, 4>(x, res, gamma, h, y, y8, scale8, rstd, rows, C, group, eps, s) : rms_fwd<float, 1>(x, res, gamma, h, y, y8, scale8, rstd, rows, C, group, eps, s);
}

int launch_add_rmsnorm_bwd(int prec, const void *dy, const void *dh, const void *h, const void *gamma, const float *rstd, void *dx, float *dgamma, float *scratch,
                           int rows, int C, Launch s) {
    const int vec = prec == P_BF16 ? 8 : 4;
    const bool v = C % vec == 0 && vec_ok(dy) && vec_ok(dh) && vec_ok(h) && vec_ok(gamma) && vec_ok(dx) && vec_ok(scratch);
    if (prec == P_BF16)
        return v ? rms_bwd<bf16, 8>(dy, dh, h, gamma, rstd, dx, dgamma, scratch, rows, C, s) : rms_bwd<bf16, 1>(dy, dh, h, gamma, rstd, dx, dgamma, scratch, rows, C, s);
    return v ? rms_bwd<float, 4>(dy, dh, h, gamma, rstd, dx, dgamma, scratch, rows, C, s) : rms_bwd<float, 1>(dy, dh, h, gamma, rstd, dx, dgamma, scratch, rows, C, s);
}

}  // namespace ddg

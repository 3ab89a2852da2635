// Root-mean-square norms after and before a block, with the block's gate and the residual's scale between them.
//
//   forward    r1 = 1 / sqrt(mean(b^2) + eps);  u = b r1 post;  h = alpha res + gate u
//              r2 = 1 / sqrt(mean(h^2) + eps);  y = h r2 pre, and / or its 8-bit codes (act8.cuh)
//   backward   t = dh + r2 (pre dy - h r2^2 mean(pre dy h))             the gradient of h
//              dres = alpha t;  dgate = sum over the gate's rows of t u
//              db = r1 (post gate t - b r1^2 mean(post gate t b));  dpost = sum gate t b r1;  dpre = sum dy h r2
//
// Bound by memory: forward b and res are read, h and y (or codes) written; backward dy, dh, b and h are read, db and dres
// written.  The two means of the backward pass, of which the second contains the first, come out of one reduction: with
// w = post gate b,
//   sum w t = sum w (dh + r2 pre dy) - r2^3 mean(pre dy h) sum w h,
// and the largest |y|, for the codes, is r2 times the largest |h pre|, which is known with the second norm's sum.
//
// From 296 rows on resident blocks walk the rows, which come through shared memory (row_ring.cuh): a row's reductions cost
// each of its warps some hundred cycles, so that few warps a row and two to eight rows at a time on an SM are faster than a row per
// SM, and arithmetic on pairs (f32x2.cuh) takes half the instructions.  Fewer rows, and rows that one warp holds, stay in
// registers.  Measured (bf16): 8192 x 4096 forward 49.0 us (5.5 TB/s), to codes 43.6 us (5.4 TB/s), backward with the folding
// kernel 75.8 us (5.3 TB/s); with a row in registers 87, 104 and 146 us.  8192 x 1021: 25, 29 and 46 us; 30000 x 256: 13, 14 and
// 26 us.  With a gate per row, which no copy brings ahead, 8192 x 4096 takes 60 us forward and 188 backward.
#include <algorithm>

#include "act8.cuh"
#include "cluster.cuh"
#include "common.cuh"
#include "lm_ops.h"
#include "row_io.cuh"
#include "row_ring.cuh"

namespace ddg {

namespace {

template <typename T, int VEC, int ITER, bool SHIFT>
__global__ void __launch_bounds__(rms_max_threads(VEC, ITER), ITER <= 2 ? 2 : 1)
block_norm_fwd_kernel(const T *b, const T *res, const T *__restrict__ gate, const T *__restrict__ post, const T *__restrict__ pre, T *h, T *y, int8_t *__restrict__ q,
                      float *__restrict__ scale, float *__restrict__ rstd_post, float *__restrict__ rstd_pre, int rows, int C, int pitch, int tpr, int span, float alpha, float eps) {
    __shared__ float red[32];
    pdl_launch();
    pdl_wait();
    const bool one_warp = tpr == 32;
    const int t = one_warp ? (threadIdx.x & 31) : threadIdx.x;
    const int row = one_warp ? blockIdx.x * (blockDim.x >> 5) + (threadIdx.x >> 5) : blockIdx.x;
    if (row >= rows) return;  // whole warps, and only where a row is one warp's
    const size_t at = (size_t)row * C;
    const int phase = SHIFT ? (int)(at % VEC) : 0;
    const T *gate_row = gate ? gate + (size_t)(row / span) * C : nullptr;
    RawRow<T, VEC, ITER, SHIFT> rb, rr;
    float v[ITER][VEC];
    float ss = 0.f;
    rb.load(b + at, t, tpr, C, phase);
    rr.load(res + at, t, tpr, C, phase);
#pragma unroll
    for (int i = 0; i < ITER; ++i) {
        const int c = (i * tpr + t) * VEC - phase;
        if (c < C) {
#pragma unroll
            for (int j = 0; j < VEC; ++j) ss = fmaf(rb.at(i, j), rb.at(i, j), ss);
        }
    }
    ss = row_reduce<false>(ss, one_warp, red);
    const float r1 = rsqrtf(ss / (float)C + eps);
    ss = 0.f;
#pragma unroll
    for (int i = 0; i < ITER; ++i) {
        const int c = (i * tpr + t) * VEC - phase;
        if (c < C) {
            float w[VEC], g[VEC];
            rms_gamma<T, VEC, SHIFT>(post, c, C, w);
            if (gate) rms_gamma<T, VEC, SHIFT>(gate_row, c, C, g);
#pragma unroll
            for (int j = 0; j < VEC; ++j) {
                const float u = rb.at(i, j) * r1 * w[j];
                v[i][j] = fmaf(alpha, rr.at(i, j), gate ? g[j] * u : u);
            }
            rms_store<T, VEC, SHIFT>(h + at, c, C, v[i]);
#pragma unroll
            for (int j = 0; j < VEC; ++j) ss = fmaf(v[i][j], v[i][j], ss);
        } else {
#pragma unroll
            for (int j = 0; j < VEC; ++j) v[i][j] = 0.f;
        }
    }
    ss = row_reduce<false>(ss, one_warp, red);
    const float r2 = rsqrtf(ss / (float)C + eps);
    if (t == 0) {
        if (rstd_post) rstd_post[row] = r1;
        if (rstd_pre) rstd_pre[row] = r2;
    }
    uint32_t top = 0;
#pragma unroll
    for (int i = 0; i < ITER; ++i) {
        const int c = (i * tpr + t) * VEC - phase;
        if (c < C) {
            float w[VEC];
            rms_gamma<T, VEC, SHIFT>(pre, c, C, w);
#pragma unroll
            for (int j = 0; j < VEC; ++j) {
                v[i][j] = v[i][j] * r2 * w[j];
                top = max(top, __float_as_uint(v[i][j]) & 0x7fffffffu);
            }
            if (y) rms_store<T, VEC, SHIFT>(y + at, c, C, v[i]);
        }
    }
    if (!q) return;
    // finite magnitudes below infinity as numbers; infinity and NaN stay above them as bits, which fmaxf would lose
    top = __reduce_max_sync(0xffffffffu, top);
    if (!one_warp) {
        uint32_t *bits = reinterpret_cast<uint32_t *>(red);
        const int nw = blockDim.x >> 5, lane = threadIdx.x & 31;
        __syncthreads();
        if (lane == 0) bits[threadIdx.x >> 5] = top;
        __syncthreads();
        top = __reduce_max_sync(0xffffffffu, lane < nw ? bits[lane] : 0u);
    }
    float s;
    const Act8Row code = act8_row(top, s);
    if (t == 0) scale[row] = s;
    int8_t *to = q + (size_t)row * pitch;
#pragma unroll
    for (int i = 0; i < ITER; ++i) {
        const int c = (i * tpr + t) * VEC - phase;
        if (c < C) {
            if (SHIFT) {
#pragma unroll
                for (int j = 0; j < VEC; ++j)
                    if (c + j >= 0 && c + j < C) to[c + j] = (int8_t)act8_code(v[i][j], code);
            } else {
                act8_store<kNear, VEC>(to + c, v[i], code);
            }
        }
    }
    for (int c = C + t; c < pitch; c += tpr) to[c] = 0;
}

struct BlockNormFwd {
    const void *b, *res, *gate, *post, *pre;
    void *h, *y;
    int8_t *q;
    float *scale, *rstd_post, *rstd_pre;
    int rows, C, pitch, span;
    float alpha, eps;
};

// The same for many rows: resident blocks walk stretches of them, the rows ahead on their way through shared memory.
// FULL: the block's threads have just the row's columns: no masks (8192 x 8192 95.5 us, 99.0 with them; to codes 8192 x 6144 72,
// 60 with them, for want of registers: not there).
template <typename T, int VEC, int ITER, bool CODES, bool FULL>
__global__ void __launch_bounds__(512, 1) block_norm_fwd_ring_kernel(const __grid_constant__ BlockNormFwd g, const __grid_constant__ RingShape shape) {
    extern __shared__ __align__(16) uint8_t ring_smem[];
    __shared__ uint64_t full[kRingMostStages];
    __shared__ __align__(16) float red[6][32];
    __shared__ int flags[2];
    const int threads = blockDim.x, t = threadIdx.x, C = g.C;
    __shared__ const uint8_t *list[2];
    RowRing<2> ring(shape, smem_u32(ring_smem), full, flags, list, {g.b, g.res});
    if (t == 0) ring.init();
    if (t < 32) {
#pragma unroll
        for (int k = 0; k < 6; ++k) red[k][t] = 0.f;
    }
    __syncthreads();
    pdl_launch();
    pdl_wait();
    const int first = (int)((long)g.rows * blockIdx.x / gridDim.x), last = (int)((long)g.rows * (blockIdx.x + 1) / gridDim.x);
    for (int row = first; row < min(first + shape.stages, last); ++row) ring.copy(row, -1);
    constexpr int P = VEC * ITER / 2, G = kGroup<VEC>;  // pairs of a thread, of a group
    typedef Share<T, VEC, ITER> Row;
    Row pre;
    F2 pg[P];   // gamma_post times the gate
    pre.load((const T *)g.pre, C, threads);
    int left = 0;  // rows that pg is for
    const float inv_c = 1.f / (float)C;
    const F2 alpha = f2(g.alpha);
    uint32_t round = 0;
    for (int row = first; row < last; ++row) {
        if (left == 0) {
            Row w;
            w.load((const T *)g.post, C, threads);
#pragma unroll
            for (int k = 0; k < P; ++k) pg[k] = w.pair(k);
            left = 1 << 30;
            if (g.gate) {
                w.load((const T *)g.gate + (size_t)(row / g.span) * C, C, threads);
#pragma unroll
                for (int k = 0; k < P; ++k) pg[k] = pg[k] * w.pair(k);
                left = g.span - row % g.span;
            }
        }
        --left;
        const bool ok = ring.wait<T, VEC>(row);
        const size_t start = (size_t)row * C;
        const uint32_t slot_b = ring.slot(0), slot_res = ring.slot(1);
        const int phase = ring_phase(shape, row);
        ring.next();
        F2 v[P], s2 = f2(0.f);
        float sum[1];
#pragma unroll
        for (int i = 0; i < P / G; ++i) {
            F2 in[G];
            slot_load<T, VEC, FULL>(slot_b, phase, C, threads, i, in);
#pragma unroll
            for (int j = 0; j < G; ++j) {
                v[i * G + j] = in[j];
                s2 = fma2(in[j], in[j], s2);
            }
        }
        sum[0] = ok ? sum2(s2) : __int_as_float(0x7fffffff);  // a row that did not come is NaN
        ring_sum<1>(sum, threads >> 5, red, round);
        if (row > first && row - 1 + shape.stages < last) ring.copy(row - 1 + shape.stages, row);
        const float r1 = rsqrtf(fmaf(sum[0], inv_c, g.eps));
        s2 = f2(0.f);
        uint32_t top = 0;
#pragma unroll
        for (int i = 0; i < P / G; ++i) {
            F2 res[G];
            slot_load<T, VEC, FULL>(slot_res, phase, C, threads, i, res);
#pragma unroll
            for (int j = 0; j < G; ++j) {
                const int k = i * G + j;
                res[j] = fma2(alpha, res[j], v[k] * f2(r1) * pg[k]);
                s2 = fma2(res[j], res[j], s2);
                v[k] = res[j] * pre.pair(k);
                if (CODES) {
                    const float2 p = parts(v[k]);
                    top = max(top, max(__float_as_uint(p.x) & 0x7fffffffu, __float_as_uint(p.y) & 0x7fffffffu));
                }
            }
            group_store<T, VEC, FULL>((T *)g.h + start, C, threads, i, res);
        }
        sum[0] = sum2(s2);
        if (CODES) ring_sum_max(sum[0], top, threads >> 5, red, round);
        else ring_sum<1>(sum, threads >> 5, red, round);
        const float r2 = rsqrtf(fmaf(sum[0], inv_c, g.eps));
        if (t == 0) {
            if (g.rstd_post) g.rstd_post[row] = r1;
            if (g.rstd_pre) g.rstd_pre[row] = r2;
        }
#pragma unroll
        for (int k = 0; k < P; ++k) v[k] = v[k] * f2(r2);
        if (g.y) share_store<T, VEC, ITER, FULL>((T *)g.y + start, C, threads, v);
        if (!CODES) continue;
        // the largest |y| is the largest |h gamma_pre| times rstd_pre: known with the sum
        float s;
        const Act8Row code = act8_row(__float_as_uint(__uint_as_float(top) * r2) & 0x7fffffffu, s);
        if (t == 0) g.scale[row] = s;
        int8_t *to = g.q + (size_t)row * g.pitch;
        act8_share_store<kNear, VEC, ITER>(to, C, threads, v, code);
        for (int c = C + t; c < g.pitch; c += threads) to[c] = 0;
    }
    if (t == 0) ring.drain();
}

struct BlockNormBwd {
    const void *dy, *dh, *b, *h, *gate, *post, *pre;
    const float *rstd_post, *rstd_pre;
    void *db, *dres;
    float *dgate;     // nullable with gate
    float *part;      // [blocks][2][C]: shares of dpost and dpre
    float *piece;     // parts > 1: [gates * parts][C], shares of dgate
    int rows, C, span, gates;
    int parts;        // a gate's rows are worked in so many stretches
    int per_block;    // a stretch is a block's, else (rows that are one warp's) a warp's
    int several;      // a block may have more than one stretch
    float alpha;
};

// Rows [r0, r1) of a stretch.  The last gate's may be fewer than its stretches, so that some are empty.
__device__ __forceinline__ void norm_stretch(const BlockNormBwd &g, int unit, int &gate, int &r0, int &r1) {
    gate = unit / g.parts;
    const int part = unit - gate * g.parts, first = gate * g.span, len = min(g.span, g.rows - first);
    r0 = first + (int)((long)len * part / g.parts);
    r1 = first + (int)((long)len * (part + 1) / g.parts);
}

// Three sums over the threads of a row.
__device__ __forceinline__ void row_sum3(float (&v)[3], bool one_warp, float (*red)[32]) {
#pragma unroll
    for (int k = 0; k < 3; ++k) v[k] = warp_sum(v[k]);
    if (one_warp) return;
    const int nw = blockDim.x >> 5, lane = threadIdx.x & 31;
    __syncthreads();  // the row before's are read
    if (lane == 0) {
#pragma unroll
        for (int k = 0; k < 3; ++k) red[k][threadIdx.x >> 5] = v[k];
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < 3; ++k) v[k] = warp_sum(lane < nw ? red[k][lane] : 0.f);
}

// Stretches of rows that share a gate are dealt out to blocks, or to warps where a row is one warp's.  Over a stretch one sum per
// column, of t b rstd_post, gives both dgate (times gamma_post) and the stretch's share of dgamma_post (times the gate).  A row is
// written after it was read, by the threads that read it, so that db and dres may be any of the tensors read row by row.  A
// warp's next row is loaded before this one is worked on where registers allow (ITER = 1).
template <typename T, int VEC, int ITER, bool WARP>
__global__ void __launch_bounds__(WARP ? 256 : rms_max_threads(VEC, ITER), WARP && ITER == 1 ? 2 : 1) block_norm_bwd_kernel(const BlockNormBwd g) {
    constexpr bool kAhead = WARP && ITER == 1;
    constexpr int N = VEC * ITER, P = (N + 1) / 2;  // values of a thread, pairs of them (the last one's second may be no value)
    __shared__ float red[3][32];
    extern __shared__ float shares[];  // WARP: [warps][C]
    pdl_launch();
    pdl_wait();
    const int warp = threadIdx.x >> 5, warps = blockDim.x >> 5, C = g.C, pitch = (C + 3) & ~3;
    const int tpr = WARP ? 32 : blockDim.x, t = WARP ? (threadIdx.x & 31) : threadIdx.x;
    const bool own = WARP && !g.per_block;  // a stretch is the warp's
    struct Row {
        Pack<T, VEC> v[ITER];
        __device__ __forceinline__ void load(const void *from, int t, int tpr, int C) {
#pragma unroll
            for (int i = 0; i < ITER; ++i) {
                const int c = (i * tpr + t) * VEC;
#pragma unroll
                for (int j = 0; j < VEC; ++j) v[i].v[j] = from_f<T>(0.f);
                if (c < C) v[i] = *reinterpret_cast<const Pack<T, VEC> *>((const T *)from + c);
            }
        }
        __device__ __forceinline__ F2 pair(int k) const {
            if constexpr (sizeof(T) == 2 && VEC > 1) return bf16_pair(reinterpret_cast<const uint32_t *>(&v[2 * k / VEC])[k % (VEC / 2)]);
            else return f2(to_f(v[2 * k / VEC].v[2 * k % VEC]), 2 * k + 1 < N ? to_f(v[(2 * k + 1) % N / VEC].v[(2 * k + 1) % VEC]) : 0.f);
        }
    };
    auto value = [](const F2 (&v)[P], int i) { const float2 p = parts(v[i / 2]); return i % 2 ? p.y : p.x; };
    // pairs of a thread as the element type, or as fp32 shares of a vector of C; shares through shared memory where the block's
    // warps have some of their own
    auto store = [&](const F2 (&v)[P], void *to) {
#pragma unroll
        for (int i = 0; i < ITER; ++i) {
            const int c = (i * tpr + t) * VEC;
            float o[VEC];
#pragma unroll
            for (int j = 0; j < VEC; ++j) o[j] = value(v, i * VEC + j);
            if (c < C) store_f<T, VEC>((T *)to + c, o);
        }
    };
    auto leave = [&](const F2 (&v)[P], float *to, bool joined) {
        float *mine = joined ? shares + warp * pitch : to;
#pragma unroll
        for (int i = 0; i < ITER; ++i) {
            const int c = (i * tpr + t) * VEC;
            float o[VEC];
#pragma unroll
            for (int j = 0; j < VEC; ++j) o[j] = value(v, i * VEC + j);
            if (c < C) store_share<VEC>(mine + c, o);
        }
        if (joined) {
            __syncthreads();
            for (int c = threadIdx.x; c < C; c += blockDim.x) {
                float sum = shares[c];
                for (int w = 1; w < warps; ++w) sum += shares[w * pitch + c];
                to[c] = sum;
            }
            __syncthreads();
        }
    };
    F2 a_post[P], a_pre[P], a_unit[P], pg[P];
    Row pre;
    pre.load(g.pre, t, tpr, C);
#pragma unroll
    for (int k = 0; k < P; ++k) a_post[k] = a_pre[k] = f2(0.f);
    const float inv_c = 1.f / (float)C;
    const int units = g.gates * g.parts, walkers = own ? gridDim.x * warps : gridDim.x;
    for (int unit = own ? blockIdx.x * warps + warp : blockIdx.x; unit < units; unit += walkers) {
        int gate, r0, r1;
        norm_stretch(g, unit, gate, r0, r1);
        const T *gate_row = g.gate ? (const T *)g.gate + (size_t)gate * C : nullptr;
        Row w;
        w.load(g.post, t, tpr, C);
#pragma unroll
        for (int k = 0; k < P; ++k) { pg[k] = w.pair(k); a_unit[k] = f2(0.f); }
        if (gate_row) {
            w.load(gate_row, t, tpr, C);
#pragma unroll
            for (int k = 0; k < P; ++k) pg[k] = pg[k] * w.pair(k);
        }
        const int step = WARP && !own ? warps : 1;
        Row dy, dh, b, h, n_dy, n_dh, n_b, n_h;
        float s1 = 0.f, s2 = 0.f, n_s1 = 0.f, n_s2 = 0.f;
        auto load = [&](int row, Row &dy, Row &dh, Row &b, Row &h, float &s1, float &s2) {
            const size_t at = (size_t)row * C;
            dy.load((const T *)g.dy + at, t, tpr, C);
            h.load((const T *)g.h + at, t, tpr, C);
            b.load((const T *)g.b + at, t, tpr, C);
            if (g.dh) dh.load((const T *)g.dh + at, t, tpr, C);
            s1 = g.rstd_post[row];
            s2 = g.rstd_pre[row];
        };
        int row = r0 + (WARP && !own ? warp : 0);
        if (kAhead && row < r1) load(row, n_dy, n_dh, n_b, n_h, n_s1, n_s2);
        for (; row < r1; row += step) {
            if (kAhead) {
                dy = n_dy; dh = n_dh; b = n_b; h = n_h; s1 = n_s1; s2 = n_s2;
                if (row + step < r1) load(row + step, n_dy, n_dh, n_b, n_h, n_s1, n_s2);
            } else {
                load(row, dy, dh, b, h, s1, s2);
            }
            F2 q0 = f2(0.f), q1 = f2(0.f), q2 = f2(0.f);
#pragma unroll
            for (int k = 0; k < P; ++k) {
                const F2 w2 = pre.pair(k) * dy.pair(k), wb = pg[k] * b.pair(k), hk = h.pair(k);
                const F2 base = g.dh ? fma2(f2(s2), w2, dh.pair(k)) : f2(s2) * w2;
                q0 = fma2(w2, hk, q0);
                q1 = fma2(wb, base, q1);
                q2 = fma2(wb, hk, q2);
            }
            float sum[3] = {sum2(q0), sum2(q1), sum2(q2)};
            row_sum3(sum, WARP, red);
            const float c2 = sum[0] * inv_c * s2 * s2 * s2, c1 = (sum[1] - c2 * sum[2]) * inv_c * s1 * s1;
            F2 o_res[P], o_b[P];
#pragma unroll
            for (int k = 0; k < P; ++k) {
                const F2 x = b.pair(k) * f2(s1), d = dy.pair(k), ds = pre.pair(k) * d, hk = h.pair(k);
                const F2 base = g.dh ? fma2(f2(s2), ds, dh.pair(k)) : f2(s2) * ds;
                const F2 tt = fma2(f2(-c2), hk, base);
                a_unit[k] = fma2(tt, x, a_unit[k]);
                a_pre[k] = fma2(d, hk * f2(s2), a_pre[k]);
                o_b[k] = fma2(pg[k], f2(s1) * tt, f2(-c1) * x);
                o_res[k] = f2(g.alpha) * tt;
            }
            store(o_res, (T *)g.dres + (size_t)row * C);
            store(o_b, (T *)g.db + (size_t)row * C);
        }
        if (gate_row) w.load(gate_row, t, tpr, C);
#pragma unroll
        for (int k = 0; k < P; ++k) a_post[k] = gate_row ? fma2(w.pair(k), a_unit[k], a_post[k]) : a_post[k] + a_unit[k];
        if (g.dgate) {
            w.load(g.post, t, tpr, C);
#pragma unroll
            for (int k = 0; k < P; ++k) a_unit[k] = a_unit[k] * w.pair(k);
            leave(a_unit, g.parts > 1 ? g.piece + (size_t)unit * C : g.dgate + (size_t)gate * C, WARP && !own);
        }
    }
    if (WARP) __syncthreads();
    leave(a_post, g.part + (size_t)blockIdx.x * 2 * C, WARP);
    leave(a_pre, g.part + (size_t)blockIdx.x * 2 * C + C, WARP);
}

// The rows of a block, one after the other.
struct NormRows {
    const BlockNormBwd &g;
    int unit, row, end;
    __device__ __forceinline__ explicit NormRows(const BlockNormBwd &a) : g(a), unit(blockIdx.x) { enter(); }
    __device__ __forceinline__ bool more() const { return unit < g.gates * g.parts; }
    __device__ __forceinline__ void enter() {
        for (; more(); unit += gridDim.x) {
            int gate;
            norm_stretch(g, unit, gate, row, end);
            if (row < end) return;
        }
    }
    __device__ __forceinline__ void next() {
        if (++row < end) return;
        unit += gridDim.x;
        enter();
    }
};

// The same for many wide rows: stretches of rows that share a gate are dealt out to resident blocks, the rows ahead on their
// way through shared memory.
// FULL: the block's threads have just the row's columns: no masks (8192 x 8192 148 us, 155 with them).
template <typename T, int VEC, int ITER, bool FULL>
__global__ void __launch_bounds__(512, 1) block_norm_bwd_ring_kernel(const __grid_constant__ BlockNormBwd g, const __grid_constant__ RingShape shape) {
    extern __shared__ __align__(16) uint8_t ring_smem[];
    __shared__ uint64_t full[kRingMostStages];
    __shared__ __align__(16) float red[6][32];
    __shared__ int flags[2];
    const int threads = blockDim.x, t = threadIdx.x, C = g.C;
    // share of dgamma_post over several stretches: [C], a thread its own columns
    float *const a_post = g.several ? reinterpret_cast<float *>(ring_smem + (size_t)shape.stages * 4 * shape.slot_bytes) : nullptr;
    if (a_post)
        for (int c = t; c < C; c += blockDim.x) a_post[c] = 0.f;  // (a barrier follows)
    __shared__ const uint8_t *list[4];
    RowRing<4> ring(shape, smem_u32(ring_smem), full, flags, list, {g.dy, g.h, g.b, g.dh});
    if (t == 0) ring.init();
    if (t < 32) {
#pragma unroll
        for (int k = 0; k < 6; ++k) red[k][t] = 0.f;
    }
    __syncthreads();
    pdl_launch();
    pdl_wait();
    NormRows ahead(g);
    for (int i = 0; i < shape.stages && ahead.more(); ++i, ahead.next()) ring.copy(ahead.row, -1);
    constexpr int P = VEC * ITER / 2, G = kGroup<VEC>;  // pairs of a thread, of a group
    typedef Share<T, VEC, ITER> Row;
    F2 a_pre[P], a_unit[P], pg[P];  // pg: gamma_post times the gate
#pragma unroll
    for (int k = 0; k < P; ++k) a_pre[k] = a_unit[k] = pg[k] = f2(0.f);  // (a cluster's last blocks may have no stretch)
    Row pre;
    pre.load((const T *)g.pre, C, threads);
    const float inv_c = 1.f / (float)C;
    const F2 alpha = f2(g.alpha);
    uint32_t round = 0;
    bool begun = false;  // there is a row before this one
    for (int unit = blockIdx.x; unit < g.gates * g.parts; unit += gridDim.x) {
        int gate, r0, r1;
        norm_stretch(g, unit, gate, r0, r1);
        const T *gate_row = g.gate ? (const T *)g.gate + (size_t)gate * C : nullptr;
        {
            Row w;
            w.load((const T *)g.post, C, threads);
#pragma unroll
            for (int k = 0; k < P; ++k) pg[k] = w.pair(k);
            if (gate_row) {
                w.load(gate_row, C, threads);
#pragma unroll
                for (int k = 0; k < P; ++k) pg[k] = pg[k] * w.pair(k);
            }
        }
#pragma unroll
        for (int k = 0; k < P; ++k) a_unit[k] = f2(0.f);
        float next1 = 0.f, next2 = 0.f;
        if (r0 < r1) { next1 = g.rstd_post[r0]; next2 = g.rstd_pre[r0]; }
        for (int row = r0; row < r1; ++row) {
            const float s1 = next1;
            float s2 = next2;
            ring.wait<T, VEC>(row);
            if (row + 1 < r1) { next1 = g.rstd_post[row + 1]; next2 = g.rstd_pre[row + 1]; }  // a row ahead
            const uint32_t slot_dy = ring.slot(0), slot_h = ring.slot(1), slot_b = ring.slot(2), slot_dh = ring.slot(3);
            const int phase = ring_phase(shape, row);
            const size_t start = (size_t)row * C;
            ring.next();
            F2 q0 = f2(0.f), q1 = f2(0.f), q2 = f2(0.f), dy[G], h[G], b[G], dh[G];
            auto load = [&](int i) {
                slot_load<T, VEC, FULL>(slot_dy, phase, C, threads, i, dy);
                slot_load<T, VEC, FULL>(slot_h, phase, C, threads, i, h);
                slot_load<T, VEC, FULL>(slot_b, phase, C, threads, i, b);
                if (g.dh) slot_load<T, VEC, FULL>(slot_dh, phase, C, threads, i, dh);
            };
#pragma unroll
            for (int i = 0; i < P / G; ++i) {
                load(i);
#pragma unroll
                for (int j = 0; j < G; ++j) {
                    const F2 w2 = pre.pair(i * G + j) * dy[j], w = pg[i * G + j] * b[j];
                    const F2 base = g.dh ? fma2(f2(s2), w2, dh[j]) : f2(s2) * w2;
                    q0 = fma2(w2, h[j], q0);
                    q1 = fma2(w, base, q1);
                    q2 = fma2(w, h[j], q2);
                }
            }
            float sum[3] = {sum2(q0), sum2(q1), sum2(q2)};
            ring_sum<3>(sum, threads >> 5, red, round);
            if (ring.lost_by(row)) s2 = __int_as_float(0x7fffffff);  // a row that did not come, to any thread, is NaN: all that follows has s2 in it
            if (begun && ahead.more()) {
                ring.copy(ahead.row, row);
                ahead.next();
            }
            begun = true;
            const float c2 = sum[0] * inv_c * s2 * s2 * s2, c1 = (sum[1] - c2 * sum[2]) * inv_c * s1 * s1;
#pragma unroll
            for (int i = 0; i < P / G; ++i) {
                load(i);
#pragma unroll
                for (int j = 0; j < G; ++j) {
                    const int k = i * G + j;
                    const F2 x = b[j] * f2(s1), ds = pre.pair(k) * dy[j];
                    const F2 base = g.dh ? fma2(f2(s2), ds, dh[j]) : f2(s2) * ds;
                    const F2 tt = fma2(f2(-c2), h[j], base);
                    a_unit[k] = fma2(tt, x, a_unit[k]);
                    a_pre[k] = fma2(dy[j], h[j] * f2(s2), a_pre[k]);
                    b[j] = fma2(pg[k], f2(s1) * tt, f2(-c1) * x);
                    h[j] = alpha * tt;
                }
                group_store<T, VEC, FULL>((T *)g.dres + start, C, threads, i, h);
                group_store<T, VEC, FULL>((T *)g.db + start, C, threads, i, b);
            }
        }
        // The stretch's one sum times the gate is its share of dgamma_post; times gamma_post, dgate's.  With one gate for all rows
        // both products are left to the folding kernel.
        if (g.gates > 1) {
            Row w;
            if (gate_row) w.load(gate_row, C, threads);
#pragma unroll
            for (int k = 0; k < P; ++k) {
                const F2 v = gate_row ? w.pair(k) * a_unit[k] : a_unit[k];
                if (a_post) {
                    const int c = VEC > 1 ? ((2 * k / VEC) * threads + t) * VEC + 2 * k % VEC : 2 * k * threads + t, d = VEC > 1 ? c + 1 : c + threads;  // columns of the pair
                    const float2 p = parts(v);
                    if (c < C) a_post[c] += p.x;
                    if (d < C) a_post[d] += p.y;
                } else {
                    pg[k] = v;  // the block's only stretch: pg has done its work
                }
            }
            if (g.dgate) {
                w.load((const T *)g.post, C, threads);
#pragma unroll
                for (int k = 0; k < P; ++k) a_unit[k] = a_unit[k] * w.pair(k);
                share_store_f32<VEC, ITER>(g.parts > 1 ? g.piece + (size_t)unit * C : g.dgate + (size_t)gate * C, C, threads, a_unit);
            }
        }
    }
    if (t == 0) ring.drain();
    // The block's shares of the two sums over all rows take the ring's place; the cluster's blocks add theirs up, a slice of the
    // columns each, blocks in index order.
    __syncthreads();
    float *const mine = reinterpret_cast<float *>(ring_smem);
    const int pitch = (C + 3) & ~3;
    if (a_post) {
        for (int c = t; c < C; c += threads) mine[c] = a_post[c];  // (another place: the stages are in front of it)
    } else {
        share_store_f32<VEC, ITER>(mine, C, threads, g.gates > 1 ? pg : a_unit);
    }
    share_store_f32<VEC, ITER>(mine + pitch, C, threads, a_pre);
    cluster_sync();
    uint32_t blocks;
    asm("mov.u32 %0, %%cluster_nctarank;" : "=r"(blocks));
    const uint32_t rank = cluster_rank(), at = smem_u32(mine);
    float *const to = g.part + (size_t)(blockIdx.x / blocks) * 2 * C;
    for (int c = (int)(rank * blockDim.x) + t; c < C; c += (int)(blocks * blockDim.x)) {
        float post[8] = {}, pre_sum[8] = {};
#pragma unroll
        for (uint32_t r = 0; r < 8; ++r)
            if (r < blocks) {
                asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(post[r]) : "r"(map_rank(at + 4u * c, r)));
                asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(pre_sum[r]) : "r"(map_rank(at + 4u * (pitch + c), r)));
            }
#pragma unroll
        for (int r = 1; r < 8; ++r) { post[0] += post[r]; pre_sum[0] += pre_sum[r]; }
        to[c] = post[0];
        to[C + c] = pre_sum[0];
    }
    cluster_sync();  // no block leaves while its shares are read
}

// Shares in index order per warp, warps in index order, 32 columns per block.  blockIdx.y: dpost, dpre, then the gate's rows.
// MORE: the gates past the rows of a grid, from sum `first` on (an offset for all launches: 695 x 6736, 13 rows a gate, 60 us
// instead of 55).
// gate and post (nullable): the first shares are still to be multiplied with the one gate, for dpost, and with gamma_post, for dgate.
constexpr int kFoldMostY = 65535;
struct NormFold { const float *part, *piece; float *dpost, *dpre, *dgate; const void *gate, *post; int n, parts, C, one_gate, first; };
template <typename T, bool MORE> __global__ void __launch_bounds__(1024) block_norm_fold_kernel(const __grid_constant__ NormFold g) {
    __shared__ float fold[32][32];
    pdl_launch();
    pdl_wait();
    const int lane = threadIdx.x & 31, w = threadIdx.x >> 5, C = g.C, c = blockIdx.x * 32 + lane, what = (MORE ? g.first : 0) + blockIdx.y, gate = what - 2;
    const float *from = what < 2 ? g.part + (size_t)what * C : g.piece + (size_t)gate * g.parts * C;
    const size_t stride = what < 2 ? 2 * (size_t)C : (size_t)C;
    const int n = what < 2 ? g.n : g.parts;
    float a = 0.f;
    if (c < C) {
#pragma unroll 8
        for (int i = w; i < n; i += 32) a += from[i * stride + c];
    }
    fold[w][lane] = a;
    __syncthreads();
    if (w == 0 && c < C) {
        for (int i = 1; i < 32; ++i) a += fold[i][lane];
        if (what == 0 && g.one_gate) {
            if (g.dgate) g.dgate[c] = a * to_f(((const T *)g.post)[c]);
            if (g.gate) a *= to_f(((const T *)g.gate)[c]);
        }
        (what == 0 ? g.dpost : (what == 1 ? g.dpre : g.dgate + (size_t)gate * C))[c] = a;
    }
}

// Whether the rows go through shared memory: 16 (backward) or 32 values of a row per thread.
RingPlan norm_ring(int rows, int C, int vec, int es, bool backward) {
    // narrow rows are a warp's of the other kernel
    int iter = vec == 1 ? 8 : (backward ? 2 : 4);
    // backward, rows of 49 to 64 vectors: one per thread (100000 x 512: 141 us, 162 with two in a warp's registers; x 384: alike)
    if (backward && vec > 1 && C / vec > 48 && C / vec <= 64) iter = 1;
    if (rows < 2 * 148 || ring_threads((C + vec - 1) / vec, iter) < 64) return RingPlan{};
    return ring_plan(C, C * es, vec, iter, backward ? 4 : 2, backward ? (size_t)C * 4 : 0);
}

// How the rows of a backward pass are dealt out: `blocks` of the launch, stretches per gate, a block or a warp a stretch.
// cluster: blocks of the ring kernel that add up their shares before they leave them.
struct BwdPlan { RingPlan ring; RmsPlan row; int blocks, parts, per_block, cluster; };
BwdPlan bwd_plan(int rows, int C, int span, int vec, int es, bool ring) {
    BwdPlan p{};
    if (ring) p.ring = norm_ring(rows, C, vec, es, true);
    p.row = rms_plan(C / vec, vec > 1, 2, 256);
    const bool warp = p.ring.threads == 0 && p.row.tpr == 32;
    const int gates = (rows - 1) / span + 1, longest = std::min(span, rows);
    p.cluster = 1;
    if (p.ring.threads && p.ring.per_sm > 1) p.cluster = 2;  // (of larger clusters the GPU holds fewer blocks than of single ones)
    const int most = 148 * (p.ring.threads ? p.ring.per_sm : (warp ? 2 : std::max(1, (p.row.iter == 1 ? 1024 : 512) / p.row.threads)));
    // rounds of the resident blocks, in rows; leaving a stretch's share costs about a row
    double best = 1e30;
    if (warp) {
        p.parts = 1;
        p.per_block = 0;
        best = (double)((gates - 1) / (most * 8) + 1) * (longest + 1);
    }
    const int even = std::max(1, most / gates);
    for (int n : {1, std::min(even, longest), std::min(even + 1, longest), std::min(2 * even, longest)}) {
        const int len = (longest - 1) / n + 1, steps = warp ? (len - 1) / 8 + 1 : len;
        const double t = (double)(((long)gates * n - 1) / most + 1) * (steps + 1);
        if (t < best) { best = t; p.parts = n; p.per_block = 1; }
    }
    const long units = (long)gates * p.parts;
    p.blocks = (int)std::min<long>(most, p.per_block ? units : (units + 7) / 8);
    p.blocks = (p.blocks + p.cluster - 1) / p.cluster * p.cluster;
    return p;
}
size_t bwd_scratch(const BwdPlan &p, int rows, int C, int span) {
    return ((size_t)p.blocks * 2 + (p.parts > 1 ? (size_t)((rows - 1) / span + 1) * p.parts : 0)) * C;
}

template <typename T, int VEC, int ITER, bool FULL> int fwd_ring_as(const BlockNormFwd &g, const RingPlan &p, const Launch &s) {
    static thread_local int ready[2] = {-1, -1};
    auto kernel = g.q ? block_norm_fwd_ring_kernel<T, VEC, ITER, true, false> : block_norm_fwd_ring_kernel<T, VEC, ITER, false, FULL>;
    if (!ring_ready(kernel, ready[g.q != nullptr])) return -1;
    launch_k(kernel, std::min(g.rows, 148 * p.per_sm), p.threads, p.smem, s, g, ring_shape(g.rows, g.C * (int)sizeof(T), 2, p.smem, block8_polls()));
    return 1;
}
template <typename T, int VEC, int ITER> int fwd_ring(const BlockNormFwd &g, const RingPlan &p, const Launch &s) {
    return VEC > 1 && !g.q && p.threads * VEC * ITER == g.C ? fwd_ring_as<T, VEC, ITER, (VEC > 1)>(g, p, s) : fwd_ring_as<T, VEC, ITER, false>(g, p, s);
}
template <typename T, int VEC, bool SHIFT> int fwd_as(const BlockNormFwd &g, const Launch &s) {
    const RmsPlan p = rms_plan(rms_nvec(g.C, VEC, SHIFT), VEC > 1, 4, 128);
    auto go = [&](auto kernel) {
        launch_k(kernel, (g.rows - 1) / p.rpb + 1, p.threads, 0, s, (const T *)g.b, (const T *)g.res, (const T *)g.gate, (const T *)g.post, (const T *)g.pre, (T *)g.h, (T *)g.y, g.q,
                 g.scale, g.rstd_post, g.rstd_pre, g.rows, g.C, g.pitch, p.tpr, g.span, g.alpha, g.eps);
    };
    switch (p.iter) {
    case 1: go(block_norm_fwd_kernel<T, VEC, 1, SHIFT>); break;
    case 2: go(block_norm_fwd_kernel<T, VEC, 2, SHIFT>); break;
    case 4: go(block_norm_fwd_kernel<T, VEC, 4, SHIFT>); break;
    case 8: if (VEC == 1) { go(block_norm_fwd_kernel<T, 1, 8, false>); break; } return -1;
    case 16: if (VEC == 1) { go(block_norm_fwd_kernel<T, 1, 16, false>); break; } return -1;
    default: return -1;
    }
    return 1;
}

template <typename T, int VEC, int ITER, bool FULL> int bwd_ring(const BlockNormBwd &g, const BwdPlan &p, const Launch &s) {
    static thread_local int ready = -1;
    if (!ring_ready(block_norm_bwd_ring_kernel<T, VEC, ITER, FULL>, ready)) return -1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(p.blocks); cfg.blockDim = dim3(p.ring.threads); cfg.dynamicSmemBytes = p.ring.smem; cfg.stream = s.s;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = p.cluster;
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[1].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = s.pdl == 1 ? 2 : 1;
    cudaLaunchKernelEx(&cfg, block_norm_bwd_ring_kernel<T, VEC, ITER, FULL>, g, ring_shape(g.rows, g.C * (int)sizeof(T), 4, p.ring.smem - (g.several ? (size_t)g.C * 4 : 0), block8_polls()));
    return 1;
}

template <typename T, int VEC> int bwd_as(BlockNormBwd &g, bool ring, float *scratch, float *dpost, float *dpre, const Launch &s) {
    const BwdPlan p = bwd_plan(g.rows, g.C, g.span, VEC, sizeof(T), ring);
    g.parts = p.parts; g.per_block = p.per_block;
    g.part = scratch;
    g.piece = scratch + (size_t)p.blocks * 2 * g.C;
    const size_t smem = p.row.tpr == 32 ? (size_t)8 * ((g.C + 3) & ~3) * sizeof(float) : 0;
    auto go = [&](auto kernel) { launch_k(kernel, p.blocks, p.row.threads, smem, s, g); };
    if (p.ring.threads) {
        g.several = (long)g.gates * g.parts > p.blocks;  // (with one gate never: its stretches are no more than the blocks)
        constexpr int ITER = VEC == 1 ? 8 : 2, SHORT = VEC == 1 ? 8 : 1;
        const bool fills = VEC > 1 && p.ring.threads * VEC * p.ring.iter == g.C;
        int r;
        if (p.ring.iter == ITER) r = fills ? bwd_ring<T, VEC, ITER, (VEC > 1)>(g, p, s) : bwd_ring<T, VEC, ITER, false>(g, p, s);
        else r = fills ? bwd_ring<T, VEC, SHORT, (VEC > 1)>(g, p, s) : bwd_ring<T, VEC, SHORT, false>(g, p, s);
        if (r < 0) return r;
    } else if (p.row.tpr == 32) {
        if (p.row.iter == 1) go(block_norm_bwd_kernel<T, VEC, 1, true>); else go(block_norm_bwd_kernel<T, VEC, 2, true>);
    } else {
        switch (p.row.iter) {
        case 1: go(block_norm_bwd_kernel<T, VEC, 1, false>); break;
        case 2: go(block_norm_bwd_kernel<T, VEC, 2, false>); break;
        case 4: go(block_norm_bwd_kernel<T, VEC, 4, false>); break;
        case 8: if (VEC == 1) { go(block_norm_bwd_kernel<T, 1, 8, false>); break; } return -1;
        case 16: if (VEC == 1) { go(block_norm_bwd_kernel<T, 1, 16, false>); break; } return -1;
        default: return -1;
        }
    }
    const bool ring_one = p.ring.threads && g.gates == 1;
    const int sums = 2 + (g.dgate && p.parts > 1 && !ring_one ? g.gates : 0);
    NormFold fold{g.part, g.piece, dpost, dpre, g.dgate, g.gate, g.post, p.ring.threads ? p.blocks / p.cluster : p.blocks, p.parts, g.C, ring_one, 0};
    int launches = 1;
    for (; fold.first < sums; fold.first += kFoldMostY, ++launches)
        launch_k(fold.first ? block_norm_fold_kernel<T, true> : block_norm_fold_kernel<T, false>, dim3((g.C + 31) / 32, std::min(sums - fold.first, kFoldMostY)), 1024, 0, s, fold);
    return launches;
}

}  // namespace

size_t block_norm_scratch_elems(int rows, int C, int span) {
    size_t most = 0;
    for (int of : {span, rows})  // with a gate, without
        for (int vec : {1, 4, 8})
            for (int es : {2, 4})
                for (bool ring : {false, true})
                    if (C % vec == 0) most = std::max(most, bwd_scratch(bwd_plan(rows, C, of, vec, es, ring), rows, C, of));
    return most;
}

int launch_block_norm_fwd(int prec, const void *b, const void *res, const void *gate, const void *post, const void *pre, void *h, void *y, void *q, float *scale,
                          float *rstd_post, float *rstd_pre, int rows, int C, int span, float alpha, float eps, Launch s) {
    const int vec = prec == P_BF16 ? 8 : 4, es = (int)elem_size(prec);
    bool aligned = true;
    for (const void *p : {b, res, gate, post, pre, (const void *)h, (const void *)y}) aligned = aligned && vec_ok(p);
    const bool v = C % vec == 0 && aligned, shift = C % vec != 0 && aligned && rms_shift_fits(C, vec);
    const BlockNormFwd g{b, res, gate, post, pre, h, y, (int8_t *)q, scale, rstd_post, rstd_pre, rows, C, act8_pitch(C), span, alpha, eps};
    if (vec_ok(b) && vec_ok(res)) {
        const RingPlan p = norm_ring(rows, C, v ? vec : 1, es, false);
        if (p.threads) {
            if (prec == P_BF16) return v ? fwd_ring<bf16, 8, 4>(g, p, s) : fwd_ring<bf16, 1, 8>(g, p, s);
            return v ? fwd_ring<float, 4, 4>(g, p, s) : fwd_ring<float, 1, 8>(g, p, s);
        }
    }
    if (prec == P_BF16) return v ? fwd_as<bf16, 8, false>(g, s) : (shift ? fwd_as<bf16, 8, true>(g, s) : fwd_as<bf16, 1, false>(g, s));
    return v ? fwd_as<float, 4, false>(g, s) : (shift ? fwd_as<float, 4, true>(g, s) : fwd_as<float, 1, false>(g, s));
}

int launch_block_norm_bwd(int prec, const void *dy, const void *dh, const void *b, const void *h, const void *gate, const void *post, const void *pre,
                          const float *rstd_post, const float *rstd_pre, void *db, void *dres, float *dgate, float *dpost, float *dpre, float *scratch, int rows, int C,
                          int span, float alpha, Launch s) {
    if (!gate) span = rows;  // no gate is one gate for all rows
    const int vec = prec == P_BF16 ? 8 : 4;
    bool v = C % vec == 0;
    for (const void *p : {dy, dh, b, h, gate, post, pre, (const void *)db, (const void *)dres, (const void *)dgate, (const void *)scratch}) v = v && vec_ok(p);
    const bool ring = vec_ok(dy) && vec_ok(dh) && vec_ok(b) && vec_ok(h);
    BlockNormBwd g{};
    g.dy = dy; g.dh = dh; g.b = b; g.h = h; g.gate = gate; g.post = post; g.pre = pre; g.rstd_post = rstd_post; g.rstd_pre = rstd_pre;
    g.db = db; g.dres = dres; g.dgate = dgate; g.rows = rows; g.C = C; g.span = span; g.gates = (rows - 1) / span + 1; g.alpha = alpha;
    if (prec == P_BF16) return v ? bwd_as<bf16, 8>(g, ring, scratch, dpost, dpre, s) : bwd_as<bf16, 1>(g, ring, scratch, dpost, dpre, s);
    return v ? bwd_as<float, 4>(g, ring, scratch, dpost, dpre, s) : bwd_as<float, 1>(g, ring, scratch, dpost, dpre, s);
}

}  // namespace ddg

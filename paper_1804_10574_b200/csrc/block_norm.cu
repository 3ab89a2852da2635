// Root-mean-square norms after and before a block, with the block's gate and the residual's scale between them.
//
//   forward    r1 = 1 / sqrt(mean(b^2) + eps);  u = b r1 post;  h = alpha res + gate u
//              r2 = 1 / sqrt(mean(h^2) + eps);  y = h r2 pre, and / or its 8-bit codes (act8.cuh)
//   backward   t = dh + r2 (pre dy - h r2^2 mean(pre dy h))             the gradient of h
//              dres = alpha t;  dgate = sum over the gate's rows of t u
//              db = r1 (post gate t - b r1^2 mean(post gate t b));  dpost = sum gate t b r1;  dpre = sum dy h r2
//
// Bound by memory: forward b and res are read, h and y (or codes) written; backward dy, dh, b and h are read, db and dres
// written.  A row stays in its threads' registers.  The two means of the backward pass, of which the second contains the
// first, come out of one reduction: with w = post gate b,
//   sum w t = sum w (dh + r2 pre dy) - r2^3 mean(pre dy h) sum w h.
#include <algorithm>

#include "act8.cuh"
#include "common.cuh"
#include "lm_ops.h"
#include "row_io.cuh"

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
            int k[VEC];
#pragma unroll
            for (int j = 0; j < VEC; ++j) k[j] = act8_code(v[i][j], code);
            if (SHIFT || VEC == 1) {
#pragma unroll
                for (int j = 0; j < VEC; ++j)
                    if (c + j >= 0 && c + j < C) to[c + j] = (int8_t)k[j];
            } else {
#pragma unroll
                for (int j = 0; j < VEC / 4; ++j) *reinterpret_cast<uint32_t *>(to + c + 4 * j) = act8_pack4(k[4 * j], k[VEC > 1 ? 4 * j + 1 : 0], k[VEC > 1 ? 4 * j + 2 : 0], k[VEC > 1 ? 4 * j + 3 : 0]);
            }
        }
    }
    for (int c = C + t; c < pitch; c += tpr) to[c] = 0;
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
    float alpha;
};

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

// Stretches of rows that share a gate are dealt out to blocks (or warps): dgate's share stays in registers over a stretch,
// those of dpost and dpre over all of a block's.  A row is written after it was read, by the threads that read it, so that
// db and dres may be any of the tensors read row by row.
template <typename T, int VEC, int ITER, bool WARP>
__global__ void __launch_bounds__(WARP ? 256 : rms_max_threads(VEC, ITER), 1) block_norm_bwd_kernel(const BlockNormBwd g) {
    __shared__ float red[3][32];
    extern __shared__ float shares[];  // WARP: [warps][C]
    pdl_launch();
    pdl_wait();
    const int warp = threadIdx.x >> 5, warps = blockDim.x >> 5, C = g.C, pitch = (C + 3) & ~3;
    const int tpr = WARP ? 32 : blockDim.x, t = WARP ? (threadIdx.x & 31) : threadIdx.x;
    const bool own = WARP && !g.per_block;  // a stretch is the warp's
    float a_post[ITER][VEC], a_pre[ITER][VEC], a_gate[ITER][VEC];
#pragma unroll
    for (int i = 0; i < ITER; ++i)
#pragma unroll
        for (int j = 0; j < VEC; ++j) a_post[i][j] = a_pre[i][j] = 0.f;
    // a block's share of a vector of C to `to`; through shared memory where its warps have shares of their own
    auto leave = [&](float (&v)[ITER][VEC], float *to, bool joined) {
        float *mine = joined ? shares + warp * pitch : to;
#pragma unroll
        for (int i = 0; i < ITER; ++i) {
            const int c = (i * tpr + t) * VEC;
            if (c < C) store_share<VEC>(mine + c, v[i]);
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
    const int units = g.gates * g.parts, walkers = own ? gridDim.x * warps : gridDim.x;
    for (int unit = own ? blockIdx.x * warps + warp : blockIdx.x; unit < units; unit += walkers) {
        const int gate = unit / g.parts, part = unit - gate * g.parts;
        const int first = gate * g.span, len = min(g.span, g.rows - first);
        const int r0 = first + (int)((long)len * part / g.parts), r1 = first + (int)((long)len * (part + 1) / g.parts);
        const T *gate_row = g.gate ? (const T *)g.gate + (size_t)gate * C : nullptr;
#pragma unroll
        for (int i = 0; i < ITER; ++i)
#pragma unroll
            for (int j = 0; j < VEC; ++j) a_gate[i][j] = 0.f;
        for (int row = r0 + (WARP && !own ? warp : 0); row < r1; row += WARP && !own ? warps : 1) {
            const size_t at = (size_t)row * C;
            RawRow<T, VEC, ITER, false> dy, dh, b, h;
            dy.load((const T *)g.dy + at, t, tpr, C, 0);
            h.load((const T *)g.h + at, t, tpr, C, 0);
            b.load((const T *)g.b + at, t, tpr, C, 0);
            if (g.dh) dh.load((const T *)g.dh + at, t, tpr, C, 0);
            const float s1 = g.rstd_post[row], s2 = g.rstd_pre[row];
            float sum[3] = {0.f, 0.f, 0.f};
#pragma unroll
            for (int i = 0; i < ITER; ++i) {
                const int c = (i * tpr + t) * VEC;
                if (c < C) {
                    float wg[VEC], wp[VEC], wr[VEC];
                    load_f<T, VEC>((const T *)g.post + c, wp);
                    load_f<T, VEC>((const T *)g.pre + c, wr);
                    if (gate_row) load_f<T, VEC>(gate_row + c, wg);
#pragma unroll
                    for (int j = 0; j < VEC; ++j) {
                        const float w2 = wr[j] * dy.at(i, j), w = wp[j] * (gate_row ? wg[j] : 1.f) * b.at(i, j);
                        const float base = fmaf(s2, w2, g.dh ? dh.at(i, j) : 0.f);
                        sum[0] = fmaf(w2, h.at(i, j), sum[0]);
                        sum[1] = fmaf(w, base, sum[1]);
                        sum[2] = fmaf(w, h.at(i, j), sum[2]);
                    }
                }
            }
            row_sum3(sum, WARP, red);
            const float c2 = sum[0] / (float)C * s2 * s2 * s2, c1 = (sum[1] - c2 * sum[2]) / (float)C * s1 * s1;
#pragma unroll
            for (int i = 0; i < ITER; ++i) {
                const int c = (i * tpr + t) * VEC;
                if (c < C) {
                    float wg[VEC], wp[VEC], wr[VEC], o_res[VEC], o_b[VEC];
                    load_f<T, VEC>((const T *)g.post + c, wp);
                    load_f<T, VEC>((const T *)g.pre + c, wr);
                    if (gate_row) load_f<T, VEC>(gate_row + c, wg);
#pragma unroll
                    for (int j = 0; j < VEC; ++j) {
                        const float base = fmaf(s2, wr[j] * dy.at(i, j), g.dh ? dh.at(i, j) : 0.f);
                        const float tt = fmaf(-c2, h.at(i, j), base), unit_b = b.at(i, j) * s1, du = gate_row ? wg[j] * tt : tt;
                        o_res[j] = g.alpha * tt;
                        o_b[j] = s1 * fmaf(wp[j], du, -c1 * b.at(i, j));
                        a_gate[i][j] = fmaf(tt, unit_b * wp[j], a_gate[i][j]);
                        a_post[i][j] = fmaf(du, unit_b, a_post[i][j]);
                        a_pre[i][j] = fmaf(dy.at(i, j), h.at(i, j) * s2, a_pre[i][j]);
                    }
                    store_f<T, VEC>((T *)g.dres + at + c, o_res);
                    store_f<T, VEC>((T *)g.db + at + c, o_b);
                }
            }
        }
        if (g.dgate) leave(a_gate, g.parts > 1 ? g.piece + (size_t)unit * C : g.dgate + (size_t)gate * C, WARP && !own);
    }
    if (WARP) __syncthreads();
    leave(a_post, g.part + (size_t)blockIdx.x * 2 * C, WARP);
    leave(a_pre, g.part + (size_t)blockIdx.x * 2 * C + C, WARP);
}

// Shares in index order per warp, warps in index order, 32 columns per block.  blockIdx.y: dpost, dpre, then the gate's rows.
__global__ void __launch_bounds__(1024) block_norm_fold_kernel(const float *__restrict__ part, const float *__restrict__ piece, int blocks, int parts, float *__restrict__ dpost,
                                                               float *__restrict__ dpre, float *__restrict__ dgate, int C) {
    __shared__ float fold[32][32];
    pdl_launch();
    pdl_wait();
    const int lane = threadIdx.x & 31, w = threadIdx.x >> 5, c = blockIdx.x * 32 + lane, what = blockIdx.y, gate = what - 2;
    const float *from = what < 2 ? part + (size_t)what * C : piece + (size_t)gate * parts * C;
    const size_t stride = what < 2 ? 2 * (size_t)C : (size_t)C;
    const int n = what < 2 ? blocks : parts;
    float a = 0.f;
    if (c < C) {
#pragma unroll 8
        for (int i = w; i < n; i += 32) a += from[i * stride + c];
    }
    fold[w][lane] = a;
    __syncthreads();
    if (w == 0 && c < C) {
        for (int i = 1; i < 32; ++i) a += fold[i][lane];
        (what == 0 ? dpost : (what == 1 ? dpre : dgate + (size_t)gate * C))[c] = a;
    }
}

// How the rows of a backward pass are dealt out: `blocks` of the launch, stretches per gate, a block or a warp a stretch.
struct BwdPlan { RmsPlan row; int blocks, parts, per_block; };
BwdPlan bwd_plan(int rows, int C, int span, int vec) {
    BwdPlan p;
    p.row = rms_plan(C / vec, vec > 1, 2, 256);
    const bool warp = p.row.tpr == 32;
    const int gates = (rows - 1) / span + 1;
    const int most = 148 * (warp ? 2 : std::max(1, (p.row.iter == 1 ? 1024 : 512) / p.row.threads));
    // rounds of the resident blocks, in rows; leaving a stretch's share costs about a row
    double best = 1e30;
    if (warp) {
        p.parts = 1;
        p.per_block = 0;
        best = (double)((gates - 1) / (most * 8) + 1) * (std::min(span, rows) + 1);
    }
    for (int n = 1; n <= std::min(std::min(span, rows), 2 * most / gates + 1); ++n) {
        const int len = (std::min(span, rows) - 1) / n + 1, steps = warp ? (len - 1) / 8 + 1 : len;
        const double t = (double)(((long)gates * n - 1) / most + 1) * (steps + 1);
        if (t < best) { best = t; p.parts = n; p.per_block = 1; }
    }
    const long units = (long)gates * p.parts;
    p.blocks = (int)std::min<long>(most, p.per_block ? units : (units + 7) / 8);
    return p;
}
size_t bwd_scratch(const BwdPlan &p, int rows, int C, int span) {
    return ((size_t)p.blocks * 2 + (p.parts > 1 ? (size_t)((rows - 1) / span + 1) * p.parts : 0)) * C;
}

template <typename T, int VEC, bool SHIFT>
int fwd_as(const void *b, const void *res, const void *gate, const void *post, const void *pre, void *h, void *y, void *q, float *scale, float *rstd_post,
           float *rstd_pre, int rows, int C, int span, float alpha, float eps, const Launch &s) {
    const RmsPlan p = rms_plan(rms_nvec(C, VEC, SHIFT), VEC > 1, 4, 128);
    auto go = [&](auto kernel) {
        launch_k(kernel, (rows - 1) / p.rpb + 1, p.threads, 0, s, (const T *)b, (const T *)res, (const T *)gate, (const T *)post, (const T *)pre, (T *)h, (T *)y, (int8_t *)q,
                 scale, rstd_post, rstd_pre, rows, C, act8_pitch(C), p.tpr, span, alpha, eps);
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

template <typename T, int VEC> int bwd_as(BlockNormBwd &g, float *scratch, float *dpost, float *dpre, const Launch &s) {
    const BwdPlan p = bwd_plan(g.rows, g.C, g.span, VEC);
    g.parts = p.parts; g.per_block = p.per_block;
    g.part = scratch;
    g.piece = scratch + (size_t)p.blocks * 2 * g.C;
    const size_t smem = p.row.tpr == 32 ? (size_t)8 * ((g.C + 3) & ~3) * sizeof(float) : 0;
    auto go = [&](auto kernel) { launch_k(kernel, p.blocks, p.row.threads, smem, s, g); };
    if (p.row.tpr == 32) {
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
    launch_k(block_norm_fold_kernel, dim3((g.C + 31) / 32, 2 + (g.dgate && p.parts > 1 ? g.gates : 0)), 1024, 0, s, (const float *)g.part, (const float *)g.piece, p.blocks,
             p.parts, dpost, dpre, g.dgate, g.C);
    return 2;
}

}  // namespace

size_t block_norm_scratch_elems(int rows, int C, int span) {
    size_t most = bwd_scratch(bwd_plan(rows, C, span, 1), rows, C, span);
    for (int vec : {4, 8})
        if (C % vec == 0) most = std::max(most, bwd_scratch(bwd_plan(rows, C, span, vec), rows, C, span));
    return most;
}

int launch_block_norm_fwd(int prec, const void *b, const void *res, const void *gate, const void *post, const void *pre, void *h, void *y, void *q, float *scale,
                          float *rstd_post, float *rstd_pre, int rows, int C, int span, float alpha, float eps, Launch s) {
    const int vec = prec == P_BF16 ? 8 : 4;
    bool aligned = true;
    for (const void *p : {b, res, gate, post, pre, (const void *)h, (const void *)y}) aligned = aligned && vec_ok(p);
    const bool v = C % vec == 0 && aligned, shift = C % vec != 0 && aligned && rms_shift_fits(C, vec);
    auto go = [&](auto f) { return f(b, res, gate, post, pre, h, y, q, scale, rstd_post, rstd_pre, rows, C, span, alpha, eps, s); };
    if (prec == P_BF16) return v ? go(fwd_as<bf16, 8, false>) : (shift ? go(fwd_as<bf16, 8, true>) : go(fwd_as<bf16, 1, false>));
    return v ? go(fwd_as<float, 4, false>) : (shift ? go(fwd_as<float, 4, true>) : go(fwd_as<float, 1, false>));
}

int launch_block_norm_bwd(int prec, const void *dy, const void *dh, const void *b, const void *h, const void *gate, const void *post, const void *pre,
                          const float *rstd_post, const float *rstd_pre, void *db, void *dres, float *dgate, float *dpost, float *dpre, float *scratch, int rows, int C,
                          int span, float alpha, Launch s) {
    const int vec = prec == P_BF16 ? 8 : 4;
    bool v = C % vec == 0;
    for (const void *p : {dy, dh, b, h, gate, post, pre, (const void *)db, (const void *)dres, (const void *)dgate, (const void *)scratch}) v = v && vec_ok(p);
    BlockNormBwd g{};
    g.dy = dy; g.dh = dh; g.b = b; g.h = h; g.gate = gate; g.post = post; g.pre = pre; g.rstd_post = rstd_post; g.rstd_pre = rstd_pre;
    g.db = db; g.dres = dres; g.dgate = dgate; g.rows = rows; g.C = C; g.span = span; g.gates = (rows - 1) / span + 1; g.alpha = alpha;
    if (prec == P_BF16) return v ? bwd_as<bf16, 8>(g, scratch, dpost, dpre, s) : bwd_as<bf16, 1>(g, scratch, dpost, dpre, s);
    return v ? bwd_as<float, 4>(g, scratch, dpost, dpre, s) : bwd_as<float, 1>(g, scratch, dpost, dpre, s);
}

}  // namespace ddg

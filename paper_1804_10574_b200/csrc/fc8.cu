// Fully connected layer on rows of 8-bit codes (act8.cuh).
//
//   forward    y_no = xs_n ws_o (sum_k xq_nk wq_ok) + b_o        32-bit integer sums, exact
//   backward   dx = dy w^;  dW = dy^T x^;  db = sum_n dy_n       w^, x^: what the codes stand for in the element type
//
// The products run on one tcgen05 kernel, CTA pairs on tiles of 256 x 256 (pair_mma.cuh); a few rows (fc8_rows.cuh) and the
// gradients of small layers (fc8_small.cuh) have kernels of their own.  What bounds it: the forward pass B in out multiply-adds of
// 8-bit integers (kind::i8, twice the rate of bf16 by the same bytes of operands), the backward pass twice as many of bf16.
// The codes are the operands of the forward pass as they lie.  For the backward pass a first kernel writes what they stand for as
// bf16 to the workspace (the codes' rows times their scales, 46 us of the 1490 that the gradients of 8192 x 4096 x 16384 take),
// beside the sums for db, and dy where TMA cannot read it.  Measured: forward 8192 x 4096 x 4096 87.6 us (3140 TOP/s), 16384 x
// 4096 x 16384 690 to 780 us (3180 to 2820, the power cap); backward, 8192 x 4096 x 16384, dx 694 us (1584 TFLOP/s), dW as fp32
// 716 us (1535), each by itself.
//
// fp32: a code is a bf16 value as it is, so that only dy times the scale (which belongs to the summed index in both products)
// has to be split, into three bf16 terms: three products where two split operands would take six.
//
// The accumulator of bf16 products truncates, so that long chains end too small (by 2.3e-3 after 2^20 products of one sign):
// where a result stays in 32 bits, chains are cut after 1024 products and the pieces added in registers, rounded to nearest;
// where it is rounded to bf16 itself, after 65536 (1.5e-4 by proportion, a twentieth of that rounding).  Integer sums are exact.
#include <algorithm>

#include "act8.cuh"
#include "common.cuh"
#include "lm_ops.h"
#include "pair_mma.cuh"

namespace ddg {

namespace {

constexpr int kStageKw = 256;                    // bytes of K of a stage: two swizzle rows, eight MMA steps
constexpr int kBlockBytes = kHalf * kStageKw;    // one operand's 128 rows
constexpr int kStageBytes = 2 * kBlockBytes;
constexpr int kStages = 192 * 1024 / kStageBytes;
constexpr int kEpiWarps = 8;                     // two per TMEM lane quarter, each half of an accumulator's columns
constexpr int kThreads = 64 + 32 * kEpiWarps;
constexpr int kSmem = kStages * kStageBytes + kEpiWarps * kOutBuf + 1024;
static_assert(kSmem + 1536 <= 227 * 1024, "with the barriers and the epilogue's columns");
constexpr int kMostPlanes = 3;
constexpr int kPieceF32 = 1024, kPieceOut = 65536;  // K values of a chain: 32-bit results, bf16 results
constexpr int kWhole = 1 << 30;                  // a chain that is not cut
constexpr int kSmallMost = 128, kSmallMostIn = 1024;  // rows and outputs, inputs of layers whose gradients are one launch
constexpr int kPairs = 74;                       // CTA pairs of the GPU: the splits of a plan (and with them the workspace) go by this number

enum Mode { kForward, kGrad };
enum Store { kBoxes, kRows };                    // results leave by a tensor map, or a line at a time

struct MmArgs {           // a product
    int M, N;                 // rows of A, rows of B (columns of the result)
    int kblocks, n_seg;       // K blocks of a segment; segments: bf16 terms of A
    int a_mn;                 // gradients: A lies with M innermost (its rows are K values) instead of K
    int a_off[kMostPlanes];   // where a segment's term starts: in K (K-major A) or in M
    int tiles_m, tiles_n, splits, group_m;
    int width;                // columns of a tile: at most 256, a multiple of 64
    int full, cut;            // tiles (times splits) of that width; the others are cut into so many parts
    int items, b_box;         // pieces of work; rows of a box of K-major B
    int piece;                // steps of the K range (K blocks times segments) of a chain (with PROMOTE)
    int tail;                 // MMA steps in a segment's last K block
    const float *row_scale, *col_scale;  // forward
    const void *bias;         // forward, nullable
    int bias_bf16;
    void *out;                // [splits][M][ld]
    int out_bf16, store, ld;
    size_t out_split;         // elements
    int box_rows;             // rows of the result's tensor map from a split to the next
    unsigned polls;           // of a bounded wait
};
// The products of a launch, both gradients or one product: the items of the first, then those of the second.
constexpr int jobs_of(int mode) { return mode == kGrad ? 2 : 1; }
template <int JOBS> struct MmJobs { MmArgs job[JOBS]; };
template <int JOBS> struct MmMaps { CUtensorMap a[JOBS], b[JOBS], out[JOBS]; };
template <int JOBS> __device__ __forceinline__ int mm_items(const MmJobs<JOBS> &all) { return JOBS == 1 ? all.job[0].items : all.job[0].items + all.job[JOBS - 1].items; }
// the product that an item belongs to; the item becomes the product's own
template <int JOBS> __device__ __forceinline__ int mm_job(const MmJobs<JOBS> &all, int &item) {
    if (JOBS == 1 || item < all.job[0].items) return 0;
    item -= all.job[0].items;
    return JOBS - 1;
}

// All tiles of a split, in bands of group_m tile rows that are walked column by column, so that the operands of the tiles in
// flight stay in the L2.  The tiles that would make a last round of the CTA pairs with few of them at work are cut into
// narrower ones.
__device__ __forceinline__ int mm_width_of(const MmArgs &g, int item) { return item < g.full ? g.width : g.width / g.cut; }
__device__ __forceinline__ int mm_split_of(const MmArgs &g, int item) {
    return g.splits == 1 ? 0 : (item < g.full ? item : g.full + (item - g.full) / g.cut) / (g.tiles_m * g.tiles_n);
}
struct MmTile { int split, m, col, width; };  // tile row, first column
__device__ __forceinline__ MmTile mm_tile(const MmArgs &g, int item) {
    const int tail = item - g.full, tile = tail < 0 ? item : g.full + tail / g.cut, part = tail < 0 ? 0 : tail % g.cut, width = mm_width_of(g, item);
    const int per = g.tiles_m * g.tiles_n, split = g.splits == 1 ? 0 : tile / per;
    unsigned r = (unsigned)(tile - split * per);
    const unsigned band = r / (unsigned)(g.group_m * g.tiles_n);
    r -= band * g.group_m * g.tiles_n;
    const unsigned rows = min(g.group_m, g.tiles_m - (int)band * g.group_m), n = r / rows;
    return MmTile{split, (int)(band * g.group_m + r - n * rows), (int)n * g.width + part * width, width};
}
// steps of the K range of a split: at most 2^22 K blocks and segments, times 148 splits, in 32 bits
__device__ __forceinline__ void mm_range(const MmArgs &g, int split, int &i0, int &i1) {
    const unsigned n = (unsigned)(g.kblocks * g.n_seg);
    i0 = 0;
    i1 = (int)n;
    if (g.splits > 1) {
        i0 = (int)(n * (unsigned)split / (unsigned)g.splits);
        i1 = (int)(n * (unsigned)(split + 1) / (unsigned)g.splits);
    }
}
__device__ __forceinline__ int mm_piece_end(const MmArgs &g, int i, int i1) { return min(i + g.piece - (int)((unsigned)i % (unsigned)g.piece), i1); }

// The scale of a row of x as a factor `by` and a power of two `up`: a sum of codes (at most 2^31) times by is finite, and so is what
// comes after it where y is.  Scales up to 2^64, all but those of rows past 10^21, are by themselves.
struct RowScale { float by, up; };
__device__ __forceinline__ RowScale row_scale_of(float s) { return s > 0x1p64f ? RowScale{s * 0x1p-64f, 0x1p64f} : RowScale{s, 1.f}; }

// 64 columns of the warp's 32 rows, v: sums as they stand in tensor memory, at columns col .. of row `row`.
// s0, s1 and b0, b1: scale and bias of the columns, a lane each; s_col: 32 floats of the warp's own.
template <int MODE>
__device__ __forceinline__ void mm_finish(const MmArgs &g, const CUtensorMap *map_out, uint32_t buf, float *v, int split, int row, int col, int lane, const RowScale &rs,
                                          float *s_col, float s0, float s1, float b0, float b1) {
    if (MODE == kForward) {
        auto spread = [&](float of_lane, auto each) {  // a register of each lane's to all rows, 32 columns
            __syncwarp();  // what stood there has been read
            s_col[lane] = of_lane;
            __syncwarp();
#pragma unroll
            for (int j = 0; j < 32; j += 4) {
                const float4 t = *reinterpret_cast<const float4 *>(s_col + j);
                each(j, t.x); each(j + 1, t.y); each(j + 2, t.z); each(j + 3, t.w);
            }
        };
#pragma unroll
        for (int q = 0; q < 2; ++q) {
            spread(q ? s1 : s0, [&](int j, float t) { v[32 * q + j] = (float)__float_as_int(v[32 * q + j]) * rs.by * t; });
            if (__any_sync(0xffffffffu, rs.up != 1.f)) {
#pragma unroll
                for (int j = 0; j < 32; ++j) v[32 * q + j] *= rs.up;
            }
            if (g.bias) spread(q ? b1 : b0, [&](int j, float t) { v[32 * q + j] += t; });
        }
    }
    const int row0 = row - lane;
    if (row0 >= g.M) return;
    if (g.store == kBoxes) {
        if (g.out_bf16) store_box(map_out, buf, lane, col, row0, v);
        else store_box_f32(map_out, buf, lane, col, row0 + split * g.box_rows, v);
        return;
    }
    if (MODE == kGrad) {  // the buffer may hold a box of the other product that is still on its way out
        if (lane == 0) asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory");
        __syncwarp();
    }
    if (g.out_bf16) {
        store_rows<true>((uint16_t *)g.out + split * g.out_split, buf, lane, row0, g.M, col, g.ld, v);
    } else {
        store_rows<false>((float *)g.out + split * g.out_split, buf, lane, row0, g.M, col, g.ld, v);
    }
}

// Gradients: B lies with N innermost, A as its product says.  PROMOTE: an accumulator holds at most `piece` steps, the epilogue
// adds the pieces.
template <int MODE, bool PROMOTE>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kThreads, 1)
mm_kernel(const __grid_constant__ MmMaps<jobs_of(MODE)> maps, const __grid_constant__ MmJobs<jobs_of(MODE)> all) {
    constexpr bool kI8 = MODE == kForward, B_MN = !kI8;
    static_assert(!kI8 || !PROMOTE, "sums of codes are exact");
    constexpr int kElem = kI8 ? 1 : 2, kw = kStageKw / kElem, kBox = 128 / kElem;
    extern __shared__ uint8_t smem_raw[];
    __shared__ uint64_t full[kStages], empty[kStages], acc_full[2], acc_empty[2], drained;
    __shared__ uint32_t tmem_holder, s_peer;
    __shared__ int abort_flag;
    __shared__ float4 s_cols[MODE == kForward ? kEpiWarps : 1][8];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t rank = cluster_rank();
    const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u;
    const Waiter wt{&abort_flag, &abort_flag, all.job[0].polls};
    if (threadIdx.x == 0) {
        for (int i = 0; i < kStages; ++i) { mbar_init(smem_u32(&full[i]), 1); mbar_init(smem_u32(&empty[i]), 1); }
        for (int i = 0; i < 2; ++i) { mbar_init(smem_u32(&acc_full[i]), 1); mbar_init(smem_u32(&acc_empty[i]), 2 * kEpiWarps); }
        mbar_init(smem_u32(&drained), 1);
        abort_flag = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 1) {
        asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&tmem_holder)), "r"(512u) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
    }
    pdl_launch();
    pdl_wait();  // nothing above touches global memory
    tc_fence_before();
    __syncthreads();
    cluster_sync();  // both CTAs' barriers are ready
    tc_fence_after();
    const uint32_t tmem = tmem_holder;
    const int n_items = mm_items(all);
    const int first = blockIdx.x >> 1, step = gridDim.x >> 1;
    // Copies into stage s of this CTA's halves of A and B: one step of the K range.
    auto load_step = [&](uint32_t s, int job, int seg, int k, int m0, int n0, int width) {
        const MmArgs &g = all.job[job];
        const CUtensorMap *map_a = &maps.a[job], *map_b = &maps.b[job];
        const int half = width / 2;  // columns of this CTA
        if (rank == 0) mbar_expect_tx(smem_u32(&full[s]), 2u * (uint32_t)(kBlockBytes + (B_MN ? (half + kBox - 1) / kBox * kBox : half) * kStageKw));
        const uint32_t bar = map_rank(smem_u32(&full[s]), 0);
        const uint32_t a = base + s * kStageBytes, b = a + kBlockBytes;
        // K-major: a box is 128 bytes of K of 128 rows.  MN-major: 64 rows of kw K values.
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            if (!kI8 && g.a_mn) tma_load_pair(a + j * (kBlockBytes / 2), map_a, bar, g.a_off[seg] + m0 + kBox * j, k);
            else tma_load_pair(a + j * (kHalf * 128), map_a, bar, g.a_off[seg] + k + kBox * j, m0);
        }
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            if (B_MN) {
                if (j * kBox < half) tma_load_pair(b + j * (kBlockBytes / 2), map_b, bar, n0 + kBox * j, k);
            } else {
                for (int r = 0; r < half; r += g.b_box) tma_load_pair(b + j * (kHalf * 128) + r * 128, map_b, bar, k + kBox * j, n0 + r);
            }
        }
    };
    uint32_t issued = 0;   // steps that this CTA's thread of the loads has issued
    bool issuer = false;   // the thread of the pair that issues the products

    if (warp == 0) {
        if (lane == 0) {  // loads
            bool ok = true;
            uint32_t s = 0, ph = 0;
            for (int item = first; item < n_items && ok; item += step) {
                int own = item;
                const int job = mm_job(all, own);
                const MmArgs &g = all.job[job];
                const MmTile t = mm_tile(g, own);
                int i0, i1;
                mm_range(g, t.split, i0, i1);
                const int m0 = t.m * kTile + (int)rank * kHalf, n0 = t.col + (int)rank * (t.width / 2);
                int kb = i0 == 0 ? 0 : i0 / g.n_seg, seg = i0 - kb * g.n_seg;
                for (int i = i0; i < i1; ++i) {
                    if (!mbar_wait(smem_u32(&empty[s]), ph ^ 1u, wt, 71)) { ok = false; break; }
                    load_step(s, job, seg, kb * kw, m0, n0, t.width);
                    ++issued;
                    if (++seg == g.n_seg) { seg = 0; ++kb; }
                    if (++s == kStages) { s = 0; ph ^= 1u; }
                }
            }
        }
        __syncwarp();
    } else if (warp == 1) {
        if (rank == 0) {
            // Products, for both CTAs: the whole warp walks a straight loop and one elected lane issues; the waits for an
            // accumulator stand outside.
            issuer = elect_one();
            // 32-bit results: fp32 (1) or int32 (2); operands: bf16 (1) of kind::f16, signed (1) of kind::i8
            const uint32_t idesc_tile = ((kI8 ? 2u : 1u) << 4) | (1u << 7) | (1u << 10) | (B_MN ? 1u << 16 : 0u) | ((uint32_t)(kTile >> 4) << 24);
            uint32_t idesc = 0;
            bool a_mn = false;
            // K-major: a step of K is 32 bytes of a swizzle row, the next 128 bytes 16 KB further.  MN-major: a step is 16 rows of
            // 128 bytes; the next 64 of the 128 M / N values lie half a block further.
            uint64_t ad0 = 0;
            const uint64_t bd0 = B_MN ? make_desc(base + kBlockBytes, 1024, 2u, kBlockBytes / 2) : make_desc(base + kBlockBytes, 1024, 2u);
            auto multiply = [&](uint32_t s, uint32_t acc, bool fresh, int steps) {
#pragma unroll
                for (int k = 0; k < 8; ++k) {
                    if (k >= steps) break;
                    const uint32_t at = s * (kStageBytes >> 4), kk = (uint32_t)((k >> 2) * (kHalf * 128 >> 4) + (k & 3) * 2);
                    const uint64_t a = ad0 + (uint64_t)(at + (a_mn ? 128u * k : kk)), b = bd0 + (uint64_t)(at + (B_MN ? 128u * k : kk));
                    if (kI8) mma_pair_i8(tmem + acc * kTile, a, b, idesc, !fresh || k > 0);
                    else mma_pair(tmem + acc * kTile, a, b, idesc, !fresh || k > 0);
                }
            };
            bool ok = true;
            uint32_t s = 0, ph = 0, u = 0;  // stage, its parity, accumulators used so far
            for (int item = first; item < n_items && ok; item += step) {
                int own = item, i0, i1;
                const MmArgs &g = all.job[mm_job(all, own)];
                const int short_from = (g.kblocks - 1) * g.n_seg;  // the last K block has g.tail steps
                mm_range(g, mm_split_of(g, own), i0, i1);
                a_mn = !kI8 && g.a_mn;
                ad0 = a_mn ? make_desc(base, 1024, 2u, kBlockBytes / 2) : make_desc(base, 1024, 2u);
                idesc = idesc_tile | (a_mn ? 1u << 15 : 0u) | ((uint32_t)(mm_width_of(g, own) >> 3) << 17);
                for (; i0 < i1; ++u) {
                    const int end = PROMOTE ? mm_piece_end(g, i0, i1) : i1;
                    const uint32_t acc = u & 1u;
                    ok = mbar_wait(smem_u32(&full[s]), ph, wt, 73) && mbar_wait(smem_u32(&acc_empty[acc]), ((u >> 1) & 1u) ^ 1u, wt, 72);
                    if (!ok) break;
                    tc_fence_after();
                    if (issuer) {
                        multiply(s, acc, true, i0 >= short_from ? g.tail : 8);
                        commit_pair(smem_u32(&empty[s]));
                    }
                    if (++s == kStages) { s = 0; ph ^= 1u; }
                    for (int i = i0 + 1; i < end; ++i) {
                        if (!mbar_wait(smem_u32(&full[s]), ph, wt, 73)) { ok = false; break; }
                        tc_fence_after();
                        if (issuer) {
                            if (i >= short_from) multiply(s, acc, false, g.tail);
                            else multiply(s, acc, false, 8);
                            commit_pair(smem_u32(&empty[s]));
                        }
                        if (++s == kStages) { s = 0; ph ^= 1u; }
                    }
                    if (!ok) break;
                    if (issuer) commit_pair(smem_u32(&acc_full[acc]));
                    i0 = end;
                }
            }
        }
        __syncwarp();
    } else {
        const int quarter = warp & 3, half = (warp - 2) >> 2;
        float *const s_col = reinterpret_cast<float *>(s_cols[MODE == kForward ? warp - 2 : 0]);
        const uint32_t buf = base + kStages * kStageBytes + (uint32_t)(warp - 2) * kOutBuf;
        uint32_t u = 0;
        bool ok = true;
        for (int item = first; item < n_items; item += step) {
            int own = item;
            const int job = mm_job(all, own);
            const MmArgs &g = all.job[job];
            const CUtensorMap *map_out = &maps.out[job];
            const MmTile t = mm_tile(g, own);
            const int row = t.m * kTile + (int)rank * kHalf + 32 * quarter + lane;
            const int col0 = t.col + half * kHalf, live = min(t.width - half * kHalf, g.N - col0);
            int pieces = 1;
            if (PROMOTE) {
                int i0, i1;
                mm_range(g, t.split, i0, i1);
                pieces = 0;
                for (int i = i0; i < i1; i = mm_piece_end(g, i, i1)) ++pieces;
            }
            float cs[4] = {}, cb[4] = {};  // loaded while the products run
            RowScale rs{0.f, 1.f};
            if (MODE == kForward) {
                rs = row_scale_of(row < g.M ? g.row_scale[row] : 0.f);
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    const int c = min(col0 + 32 * q + lane, g.N - 1);
                    cs[q] = g.col_scale[c];
                    if (g.bias) cb[q] = g.bias_bf16 ? to_f(((const bf16 *)g.bias)[c]) : ((const float *)g.bias)[c];
                }
            }
            float v[PROMOTE ? kHalf : kKBox];
            if (PROMOTE) {
#pragma unroll
                for (int j = 0; j < kHalf; ++j) v[PROMOTE ? j : 0] = 0.f;
            }
#pragma unroll 1
            for (int piece = 0; piece < pieces && ok; ++piece, ++u) {
                const uint32_t acc = u & 1u;
                ok = __all_sync(0xffffffffu, mbar_wait(smem_u32(&acc_full[acc]), (u >> 1) & 1u, wt, 74));
                if (!ok) break;
                tc_fence_after();
                const uint32_t taddr = tmem + acc * kTile + ((uint32_t)(32 * quarter) << 16) + (uint32_t)(half * kHalf);
                auto hand_back = [&]() {
                    tc_fence_before();
                    __syncwarp();
                    if (lane == 0) mbar_arrive_remote(map_rank(smem_u32(&acc_empty[acc]), 0));
                };
                if (!PROMOTE) {
                    // 64 columns at a time in a loop that is not unrolled: short code
#pragma unroll 1
                    for (int c = 0; c < kHalf; c += kKBox) {
                        if (c < live) {
#pragma unroll
                            for (int j = 0; j < kKBox; j += 32)
                                tc_ld32(taddr + (uint32_t)(c + j), reinterpret_cast<float(&)[16]>(v[j]), reinterpret_cast<float(&)[16]>(v[j + 16]));
                            tc_wait_ld();
                        }
                        if (c == kHalf - kKBox) hand_back();
                        if (c < live) mm_finish<MODE>(g, map_out, buf, v, t.split, row, col0 + c, lane, rs, s_col, c == 0 ? cs[0] : cs[2], c == 0 ? cs[1] : cs[3], c == 0 ? cb[0] : cb[2], c == 0 ? cb[1] : cb[3]);
                    }
                } else {
#pragma unroll
                    for (int c = 0; c < kHalf; c += 16) {
                        float w[16];
                        tc_ld16(taddr + (uint32_t)c, w);
                        tc_wait_ld();
#pragma unroll
                        for (int j = 0; j < 16; ++j) v[c + j] += w[j];
                    }
                    hand_back();
                }
            }
            if (!ok) {  // what this tile and the ones after it should have become
                for (int r = 0; r < 32 && row - lane + r < g.M; ++r)
                    for (int c = lane; c < live; c += 32) {
                        const size_t at = t.split * g.out_split + (size_t)(row - lane + r) * g.ld + col0 + c;
                        if (g.out_bf16) ((uint16_t *)g.out)[at] = 0x7fff; else ((uint32_t *)g.out)[at] = 0x7fffffffu;
                    }
                continue;
            }
            if (PROMOTE) {
#pragma unroll
                for (int c = 0; c < kHalf; c += kKBox)
                    if (c < live) mm_finish<MODE>(g, map_out, buf, v + (PROMOTE ? c : 0), t.split, row, col0 + c, lane, rs, s_col, 0.f, 0.f, 0.f, 0.f);
            }
        }
        if (lane == 0) asm volatile("cp.async.bulk.wait_group 0;" ::: "memory");
        __syncwarp();
    }
    tc_fence_before();
    __syncthreads();
    if (threadIdx.x == 0)
        asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(map_rank(smem_u32(&s_peer), rank ^ 1u)), "r"(issued | (abort_flag ? kGaveUp : 0u)) : "memory");
    cluster_sync();
    if (abort_flag || (s_peer & kGaveUp)) {
        // A wait of the pair ran out, so that products or copies may still be in flight; they would land in the shared memory
        // and TMEM of whoever has them next.  The products end by themselves, and after them nothing reads the stages.  A
        // step that only one of the CTAs has issued is completed by the other (any boxes of the same size will do), so that the barriers of all
        // steps complete: a step is at most kStages ahead of the products, so that no two of one stage are open.
        if (issuer) commit_pair(smem_u32(&drained));
        if (threadIdx.x == 0) mbar_drain(smem_u32(&drained), 0);
        __syncthreads();
        cluster_sync();
        if (threadIdx.x == 0) {
            const uint32_t peer = s_peer & ~kGaveUp, last = max(issued, peer);
            int item = first, left = 0, job = 0, width = 0;  // the item that a step is of: how many steps up to its end
            for (uint32_t i = 0; i < peer; ++i, --left) {
                if (i > 0 && left == 0) item += step;
                if (left == 0) {
                    int own = item, i0, i1;
                    job = mm_job(all, own);
                    mm_range(all.job[job], mm_split_of(all.job[job], own), i0, i1);
                    left = i1 - i0;
                    width = mm_width_of(all.job[job], own);
                }
                if (i >= issued) load_step(i % kStages, job, 0, 0, 0, 0, width);
            }
            if (rank == 0)
                for (uint32_t i = last > kStages ? last - kStages : 0; i < last; ++i) mbar_drain(smem_u32(&full[i % kStages]), (i / kStages) & 1u);
        }
        __syncthreads();
        cluster_sync();
    }
    // no MMA of the pair reads this CTA's shared memory or writes its TMEM any more
    if (warp == 1) {
        tc_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512u) : "memory");
    }
    cluster_sync();
}

#include "fc8_rows.cuh"

#include "fc8_small.cuh"

// ---- before the products of the backward pass ------------------------------------------------------------------------
// Codes to bf16, in rows of `plane`: times their scale, or as they are (scale nullable).
struct CodesJob { const int8_t *q; const float *scale; bf16 *dst; int rows, pitch, plane, blocks; };
// dy to bf16 terms in rows of planes * plane, zeros behind a row's columns: as it is (bf16), or times the columns' factors to
// by_col (for dx) and times the rows' to by_row (for dW), each nullable.
struct TermsJob { const void *src; bf16 *plain, *by_col, *by_row; const float *row_scale, *col_scale; int rows, cols, plane, planes, blocks; };
// sums of dy over `chunk` rows: part[row chunk][cols]
struct SumsJob { const void *src; float *part; int rows, cols, chunk, blocks, vec; };
struct PrepArgs { CodesJob codes[2]; TermsJob terms; SumsJob sums; };

__device__ __forceinline__ void prep_codes(const CodesJob &j, int block) {
    const unsigned per_row = j.pitch / 16;
    const size_t units = (size_t)j.rows * per_row;
    for (size_t i = (size_t)block * 256 + threadIdx.x; i < units; i += (size_t)j.blocks * 256) {
        const size_t row = units <= 0xffffffffu ? (unsigned)i / per_row : i / per_row;
        const int c = (int)(i - row * per_row) * 16;
        const uint4 w = *reinterpret_cast<const uint4 *>(j.q + row * j.pitch + c);
        const float s = j.scale ? j.scale[row] : 1.f;
        const uint32_t word[4] = {w.x, w.y, w.z, w.w};
        uint32_t out[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            const uint32_t x = word[k / 2] >> (16 * (k % 2));
            out[k] = pack2((float)(int8_t)x * s, (float)(int8_t)(x >> 8) * s);
        }
        st_global_32(j.dst + row * j.plane + c, out);
    }
}

constexpr int kTermCols = 256;  // columns of a row that a warp has at a time, two neighbours per lane
template <typename T> __device__ __forceinline__ void prep_terms(const TermsJob &j, int block) {
    const int lane = threadIdx.x & 31;
    const unsigned per_row = (j.plane + kTermCols - 1) / kTermCols;
    const size_t items = (size_t)j.rows * per_row;
    // a's first term; a becomes the rest.  An infinity or NaN stays in the first term alone; what the rounding alone would make
    // infinite is bf16's largest value, and the rest is the next term's.
    auto first_of = [](float &a) {
        constexpr float kMost = 0x1.fep127f;
        float h = bf16_round(a), rest = a - h;
        if (!(fabsf(h) <= kMost)) {
            if (fabsf(a) < INFINITY) { h = copysignf(kMost, a); rest = a - h; } else rest = 0.f;
        }
        a = rest;
        return h;
    };
    auto leave = [&](bf16 *to, float a, float b) {
        float ha = first_of(a), hb = first_of(b);
        for (int p = 1;; ++p) {
            *reinterpret_cast<uint32_t *>(to) = pack2(ha, hb);
            if (p >= j.planes) break;
            to += j.plane;
            ha = bf16_round(a); hb = bf16_round(b);
            a -= ha; b -= hb;
        }
    };
    for (size_t i = (size_t)block * 8 + (threadIdx.x >> 5); i < items; i += (size_t)j.blocks * 8) {
        const size_t row = items <= 0xffffffffu ? (unsigned)i / per_row : i / per_row;
        const int c0 = (int)(i - row * per_row) * kTermCols + 2 * lane;
        const T *from = (const T *)j.src + row * j.cols;
        float v[kTermCols / 64][2], cs[kTermCols / 64][2];
#pragma unroll
        for (int k = 0; k < kTermCols / 64; ++k)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const int c = c0 + 64 * k + e;
                v[k][e] = c < j.cols ? to_f(from[c]) : 0.f;
                cs[k][e] = j.by_col && c < j.cols ? j.col_scale[c] : 0.f;
            }
        const float rs = j.by_row ? j.row_scale[row] : 0.f;
        const size_t at = row * j.planes * j.plane;
#pragma unroll
        for (int k = 0; k < kTermCols / 64; ++k) {
            const int c = c0 + 64 * k;
            if (c >= j.plane) break;
            if (j.plain) *reinterpret_cast<uint32_t *>(j.plain + at + c) = pack2(v[k][0], v[k][1]);
            if (j.by_col) leave(j.by_col + at + c, c < j.cols ? v[k][0] * cs[k][0] : 0.f, c + 1 < j.cols ? v[k][1] * cs[k][1] : 0.f);
            if (j.by_row) leave(j.by_row + at + c, c < j.cols ? v[k][0] * rs : 0.f, c + 1 < j.cols ? v[k][1] * rs : 0.f);
        }
    }
}

// 64 columns of a chunk of rows per block; 8 values per thread where rows start on 16-byte boundaries, else one
template <typename T> __device__ __forceinline__ void prep_sums(const SumsJob &j, int block) {
    __shared__ float fold[32][65];
    const int groups = (j.cols + 63) / 64, chunk = block / groups, c0 = (block - chunk * groups) * 64;
    const int r0 = chunk * j.chunk, r1 = min(j.rows, r0 + j.chunk);
    if (j.vec) {
        constexpr int N = Vec16<T>::N;
        const int lanes = 64 / N, l = threadIdx.x % lanes, r = threadIdx.x / lanes, step = 256 / lanes;  // 32 (bf16) or 16 rows at a time
        float a[N] = {};
        if (c0 + l * N < j.cols) {
#pragma unroll 4
            for (int row = r0 + r; row < r1; row += step) {
                float v[N];
                load_f<T, N>((const T *)j.src + (size_t)row * j.cols + c0 + l * N, v);
#pragma unroll
                for (int k = 0; k < N; ++k) a[k] += v[k];
            }
        }
#pragma unroll
        for (int k = 0; k < N; ++k) fold[r][l * N + k] = a[k];
        __syncthreads();
        if (threadIdx.x < 64 && c0 + (int)threadIdx.x < j.cols) {
            float s = 0.f;
            for (int k = 0; k < step; ++k) s += fold[k][threadIdx.x];
            j.part[(size_t)chunk * j.cols + c0 + threadIdx.x] = s;
        }
    } else {
        const int l = threadIdx.x & 63, r = threadIdx.x >> 6;
        float a = 0.f;
        if (c0 + l < j.cols) {
#pragma unroll 4
            for (int row = r0 + r; row < r1; row += 4) a += to_f(((const T *)j.src)[(size_t)row * j.cols + c0 + l]);
        }
        fold[r][l] = a;
        __syncthreads();
        if (r == 0 && c0 + l < j.cols) j.part[(size_t)chunk * j.cols + c0 + l] = ((fold[0][l] + fold[1][l]) + fold[2][l]) + fold[3][l];
    }
}

template <typename T> __global__ void __launch_bounds__(256) fc8_prep_kernel(const __grid_constant__ PrepArgs g) {
    pdl_launch();
    pdl_wait();
    int block = blockIdx.x;
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        if (block < g.codes[k].blocks) { prep_codes(g.codes[k], block); return; }
        block -= g.codes[k].blocks;
    }
    if (block < g.terms.blocks) { prep_terms<T>(g.terms, block); return; }
    block -= g.terms.blocks;
    prep_sums<T>(g.sums, block);
}

// ---- after the products of the backward pass -------------------------------------------------------------------------
// Sums of parts, in index order: of dx and dW where their K range was split, of db (a column per thread and warp).
struct JoinJob { const float *part; void *out; size_t stride, total; int parts, ld, cols, out_bf16, vec, blocks; };
struct JoinSums { const float *part; float *db; int parts, cols; };
struct JoinArgs { JoinJob job[2]; JoinSums sums; };
__device__ __forceinline__ void join_sums(const JoinSums &j, int block) {
    __shared__ float fold[8][32];
    const int lane = threadIdx.x & 31, w = threadIdx.x >> 5, c = block * 32 + lane;
    float a = 0.f;
    if (c < j.cols) {
#pragma unroll 4
        for (int i = w; i < j.parts; i += 8) a += j.part[(size_t)i * j.cols + c];
    }
    fold[w][lane] = a;
    __syncthreads();
    if (w == 0 && c < j.cols) {
        for (int i = 1; i < 8; ++i) a += fold[i][lane];
        j.db[c] = a;
    }
}
__global__ void __launch_bounds__(256) fc8_join_kernel(const __grid_constant__ JoinArgs g) {
    pdl_launch();
    pdl_wait();
    int block = blockIdx.x, k = 0;
    for (; k < 2 && block >= g.job[k].blocks; ++k) block -= g.job[k].blocks;
    if (k == 2) { join_sums(g.sums, block); return; }
    const JoinJob &j = g.job[k];
    for (size_t i = (size_t)block * 256 + threadIdx.x; i < j.total; i += (size_t)j.blocks * 256) {  // groups of four columns
        const size_t row = i / (j.ld / 4);
        const int c = (int)(i - row * (j.ld / 4)) * 4;
        float v[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
        for (int s = 0; s < j.parts; ++s) {
            const float4 q = *reinterpret_cast<const float4 *>(j.part + s * j.stride + row * j.ld + c);
            v[0] += q.x; v[1] += q.y; v[2] += q.z; v[3] += q.w;
        }
        const size_t at = row * j.cols + c;
        if (j.vec && c + 4 <= j.cols) {
            if (j.out_bf16) store_f<bf16, 4>((bf16 *)j.out + at, v); else store_f<float, 4>((float *)j.out + at, v);
        } else {
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (c + e < j.cols) {
                    if (j.out_bf16) ((bf16 *)j.out)[at + e] = from_f<bf16>(v[e]); else ((float *)j.out)[at + e] = v[e];
                }
        }
    }
}

// ---- host side -------------------------------------------------------------------------------------------------------
int up(int v, int to) { return (v + to - 1) / to * to; }
size_t up256(size_t v) { return (v + 255) / 256 * 256; }

int sm_count() {
    int dev = 0, n = 148;
    if (cudaGetDevice(&dev) == cudaSuccess) cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev);
    return n;
}

thread_local int t_wait_polls = -1;  // polls of a bounded wait, for the calls of this thread (negative: the default)

// what a tile takes of one of 256 columns
double mm_weight(int width) { return 0.5 + 0.5 * width / kTile; }
// Columns of the tiles of M x N (times splits): at most 256, as many tiles as that takes, alike.  Where that leaves some of the
// CTA pairs that the product may count on without work, narrower ones: half of a tile's loads, A's, stay.  (Forward 768 x 4096 x
// 4096: 14.2 us with tiles of 192 columns, 16.9 with 256.)
int mm_width(int M, int N, int splits, int pairs) {
    const long rows = (long)((M + kTile - 1) / kTile) * splits;
    int best = kTile;
    double least = 1e30;
    for (int most : {kTile, 3 * kTile / 4, kTile / 2, kTile / 4}) {
        const int tiles = (N + most - 1) / most, width = ((N + tiles - 1) / tiles + kKBox - 1) / kKBox * kKBox;
        const double t = (double)((rows * tiles + pairs - 1) / pairs) * mm_weight(width);
        if (t < 0.98 * least) { least = t; best = width; }
        if (rows * tiles >= pairs) break;
    }
    return best;
}

// A way to do a product: splits of K (steps of 128 values) where the tiles alone fill the GPU badly; each costs a write and a
// read of its sums.  Seconds by 1.4 PFLOP/s and 6 TB/s.
struct MmWay { int splits, width; long items; double each, sums; };
constexpr int kMostWays = 10;
int mm_ways(int M, int N, int steps, int pairs, MmWay (&way)[kMostWays]) {
    const long rows = (M + kTile - 1) / kTile, tiles = rows * ((N + kTile - 1) / kTile);
    const int most = (int)std::max<long>(1, std::min<long>(2 * kPairs / tiles, steps / 4));
    int n = 0;
    for (int i = 1; i <= kMostWays; ++i) {  // 1 to 8, and one or two rounds of pairs
        const int splits = (int)std::min<long>(most, i <= 8 ? i : (i - 8) * kPairs / std::max<long>(1, tiles));
        if (splits < 1 || (n && splits <= way[n - 1].splits)) continue;
        MmWay &w = way[n++];
        w.splits = splits;
        w.width = mm_width(M, N, splits, pairs);
        w.items = rows * ((N + w.width - 1) / w.width) * splits;
        w.each = mm_weight(w.width) / splits * 2.0 * kTile * kTile * 128.0 * steps * kPairs / 1.4e15;
        w.sums = splits > 1 ? 8.0 * splits * M * up(N, 4) / 6e12 : 0.0;
    }
    return n;
}
// How long two products take in a launch, the longer items first, dealt out to the CTA pairs in turn, and the launch that adds up
// the splits.
double mm_time(const MmWay &a, const MmWay &b) {
    const long whole_a = a.items / kPairs, rest_a = a.items % kPairs, whole_b = b.items / kPairs, rest_b = b.items % kPairs;
    const double t = a.sums + b.sums + (a.splits > 1 || b.splits > 1 ? 3e-6 : 0.0) + whole_a * a.each + whole_b * b.each;
    if (rest_a + rest_b > kPairs) return t + a.each + b.each;
    return t + std::max(rest_a ? a.each : 0.0, rest_b ? b.each : 0.0);
}
// Both in one launch, unless they keep the pairs busy for more than eight rounds: there a launch less is nothing, and pairs out of
// step bring operands from memory twice.  (us in one / in two: 512 x 512 x 512 8.5 / 15, fp32 1000 x 512 x 2000 28 / 40, 4096 x
// 4096 x 4096 201 / 211, fp32 635 / 700; 8192 x 4096 x 4096 419 / 414, fp32 8192 x 8192 x 8192 5250 / 5120.)
bool mm_together(const MmWay &dx, const MmWay &dw) { return dx.items + dw.items <= 8 * kPairs; }
// Both gradients share the CTA pairs: each is planned for half of them.  One that is asked for alone is split the same way, so
// that its sums are the same to the last bit.
void mm_plan(const int (&sizes)[2][3], MmWay &dx, MmWay &dw) {
    MmWay way[2][kMostWays];
    int n[2];
    for (int k = 0; k < 2; ++k) n[k] = mm_ways(sizes[k][0], sizes[k][1], sizes[k][2], kPairs / 2, way[k]);
    double least = 1e30;
    for (int i = 0; i < n[0]; ++i)
        for (int j = 0; j < n[1]; ++j) {
            const double t = mm_time(way[0][i], way[1][j]);
            if (t < least) { least = t; dx = way[0][i]; dw = way[1][j]; }
        }
}

// The tiles of the last round of the CTA pairs (so many come before these), where it is not full, are halved or quartered if that
// is done sooner: half of a part's loads, A's, stay.
void mm_cut(MmArgs &g, int before, int tiles, int pairs) {
    const int rest = before + tiles > pairs ? std::min((before + tiles) % pairs, tiles) : 0;
    g.full = tiles;
    g.cut = 1;
    double least = 0.95 * mm_weight(g.width);
    for (int c = 2; c <= 4 && rest; c *= 2) {
        if (g.width % (c * kKBox) != 0) break;
        const double t = (double)((rest * c + pairs - 1) / pairs) * mm_weight(g.width / c);
        if (t < least) { least = t; g.cut = c; g.full = tiles - rest; }
    }
    g.items = g.full + (tiles - g.full) * g.cut;
}

// An operand: a row-major matrix in memory; ld: elements from a row to the next.
struct Operand { const void *ptr; int rows, cols; size_t ld; };

// One of the products of a launch: what its sizes say, with g.M, N, n_seg, splits, width and where the results go.
// most_chain: K values of a chain (with PROMOTE).
template <int MODE> struct MmLaunch {
    static constexpr int kJobs = jobs_of(MODE), kBytes = MODE == kForward ? 1 : 2, kw = kStageKw / kBytes;
    MmMaps<kJobs> maps{};
    MmJobs<kJobs> all{};
    int n = 0, items = 0;
    int pairs = sm_count() / 2;

    // last: no other product comes behind this one
    bool add(const Operand &a, const Operand &b, MmArgs g, int K, int most_chain, bool last) {
        g.kblocks = (K + kw - 1) / kw;
        g.tail = (K - (g.kblocks - 1) * kw + 32 / kBytes - 1) / (32 / kBytes);
        g.piece = most_chain / kw;
        g.tiles_m = (g.M + kTile - 1) / kTile;
        g.tiles_n = (g.N + g.width - 1) / g.width;
        g.group_m = 16;
        g.polls = block8_polls();
        const long tiles = (long)g.tiles_m * g.tiles_n * g.splits;
        if (tiles > 0x7fffffff / 16) return false;
        g.full = g.items = (int)tiles;
        g.cut = 1;
        if (last) mm_cut(g, items, (int)tiles, pairs);
        g.b_box = g.width / g.cut / 2;
        constexpr CUtensorMapDataType type = MODE == kForward ? CU_TENSOR_MAP_DATA_TYPE_UINT8 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16;
        if (!box_map(type, kBytes, a.ptr, a.rows, a.cols, a.ld, g.a_mn ? kw : kHalf, &maps.a[n]) ||
            !box_map(type, kBytes, b.ptr, b.rows, b.cols, b.ld, MODE == kGrad ? kw : g.b_box, &maps.b[n]))
            return false;
        if (g.store == kBoxes && !box_map(g.out_bf16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT32, g.out_bf16 ? 2 : 4, g.out,
                                          g.splits > 1 ? g.splits * g.box_rows : g.M, g.splits > 1 ? g.ld : g.N, g.ld, 32, &maps.out[n]))
            return false;
        all.job[n++] = g;
        items += g.items;
        return true;
    }
    template <bool PROMOTE> int run(const Launch &s) {
        static thread_local int ready_dev = -1;  // the attribute belongs to a device
        int dev = 0;
        cudaGetDevice(&dev);
        if (ready_dev != dev) {
            if (cudaFuncSetAttribute(mm_kernel<MODE, PROMOTE>, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmem) != cudaSuccess) return -1;
            ready_dev = dev;
        }
        launch_k(mm_kernel<MODE, PROMOTE>, 2 * std::min(items, pairs), kThreads, kSmem, s, maps, all);
        return 1;
    }
};

// Where the results go: by a tensor map when their rows keep to 16 bytes.  Splits' sums lie one behind the other, with room for a
// box's rows behind the last.
void mm_out(MmArgs &g, void *out, bool is_bf16, int ld) {
    g.out = out; g.out_bf16 = is_bf16; g.ld = ld;
    g.box_rows = up(g.M, 32);
    g.out_split = (size_t)g.box_rows * ld;
    g.store = ld * (is_bf16 ? 2 : 4) % 16 == 0 && (reinterpret_cast<uintptr_t>(out) & 15) == 0 ? kBoxes : kRows;
}

int rows_columns(int B) { return B <= 16 ? 16 : (B <= 32 ? 32 : (B <= 64 ? 64 : 128)); }
// CTAs that share a tile's K range: as many as run at the same time, and as leave each more codes than sums (bytes).
int rows_splits(int nt, int tiles, int in) {
    return std::max(1, std::min(std::min(kRowsMostSplits, kRowsPerSm * 2 * kPairs / tiles), in / std::max(256, 8 * nt)));
}
// Whether the outputs go on the MMA's rows.  Both ways are bound by what an SM brings in (about 95 GB/s each), which the ways of
// cutting the work up tell, in bytes; a row's sums cost as much as 2 KB.  (us with outputs / with rows of x on the MMA's rows:
// 1 x 4096 x 16384 14.8 / 24.8; 64 x 4096 x 4096 9.8 / 11.5; 200 x 16384 x 1024 13.7 / 32.4; 256 x 4096 x 16384 25.8 / 18.8.)
bool rows_fit(int B, int in, int out) {
    const int nt = rows_columns(B), sms = 2 * kPairs;
    const long tiles = (long)((out + kHalf - 1) / kHalf) * ((B + nt - 1) / nt);
    if (B <= 32) return true;
    if (B > 1024 || tiles > kRowsPerSm * sms) return false;
    const int splits = rows_splits(nt, (int)tiles, in), width = mm_width(B, out, 1, kPairs);
    const double mine = (double)((tiles * splits + sms - 1) / sms) * ((in + splits - 1) / splits) * (kHalf + nt) + 2048.0 * nt;
    const long pairs = (long)((B + kTile - 1) / kTile) * ((out + width - 1) / width);
    return mine < (double)((pairs + kPairs - 1) / kPairs) * in * (kHalf + width / 2);
}
template <int NT> int rows_launch(const CUtensorMap &w, const CUtensorMap &x, const RowsArgs &g, int tiles, const Launch &s) {
    static thread_local int ready_dev = -1;
    int dev = 0;
    cudaGetDevice(&dev);
    if (ready_dev != dev) {
        if (cudaFuncSetAttribute(fc8_rows_kernel<NT>, cudaFuncAttributeMaxDynamicSharedMemorySize, kRowsSmem) != cudaSuccess) return -1;
        ready_dev = dev;
    }
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(tiles * g.splits); cfg.blockDim = dim3(kRowsThreads); cfg.dynamicSmemBytes = kRowsSmem; cfg.stream = s.s;
    cudaLaunchAttribute attr[2];
    cfg.attrs = attr;
    if (g.splits > 1) {
        attr[cfg.numAttrs].id = cudaLaunchAttributeClusterDimension;
        attr[cfg.numAttrs].val.clusterDim.x = g.splits;
        attr[cfg.numAttrs].val.clusterDim.y = attr[cfg.numAttrs].val.clusterDim.z = 1;
        ++cfg.numAttrs;
    }
    if (s.pdl == 1) {
        attr[cfg.numAttrs].id = cudaLaunchAttributeProgrammaticStreamSerialization;
        attr[cfg.numAttrs].val.programmaticStreamSerializationAllowed = 1;
        ++cfg.numAttrs;
    }
    cudaLaunchKernelEx(&cfg, fc8_rows_kernel<NT>, w, x, g);
    return 1;
}
struct BwdPlan {
    int planes;              // bf16 terms of dy
    bool copy_dy;            // dy is not read in place: fp32, or rows that TMA cannot read
    int plane_in, plane_out; // columns of a row of codes as bf16, of a term of dy
    MmWay dx_way, dw_way;
    int ld;
    int chunk, chunks;       // rows of dy that are summed up at a time for db
    size_t x, w, dy[2], dx, dw, db, bytes;
};
BwdPlan bwd_plan(int prec, int B, int in, int out) {
    BwdPlan p{};
    p.planes = prec == P_F32 ? kMostPlanes : 1;
    p.plane_in = up(in, 64);
    p.plane_out = prec == P_F32 ? up(out, 128) : up(out, 64);  // fp32: a K block never reaches into the next term
    p.ld = up(in, 4);
    const int kw = kStageKw / 2;
    const int sizes[2][3] = {{B, in, (out + kw - 1) / kw * p.planes}, {out, in, (B + kw - 1) / kw * p.planes}};
    mm_plan(sizes, p.dx_way, p.dw_way);
    // so that a thread has 8 rows to add up (the join that the splits take adds up db's too), or some more where that saves a launch
    const int sum_rows = (out % 8 == 0 ? 128 : 32) * (p.dx_way.splits > 1 || p.dw_way.splits > 1 ? 1 : 4);
    p.chunk = B <= sum_rows ? B : std::max(std::min(sum_rows, 256), (B + 127) / 128);
    p.chunks = (B + p.chunk - 1) / p.chunk;
    size_t at = 0;
    auto take = [&](size_t bytes) { const size_t r = at; at += up256(bytes); return r; };
    p.x = take((size_t)B * p.plane_in * 2);
    p.w = take((size_t)out * p.plane_in * 2);
    for (int k = 0; k < (prec == P_F32 ? 2 : 1); ++k) p.dy[k] = take((size_t)B * p.planes * p.plane_out * 2);  // also for a bf16 dy that starts anywhere
    if (p.dx_way.splits > 1) p.dx = take((size_t)p.dx_way.splits * up(B, 32) * p.ld * 4);
    if (p.dw_way.splits > 1) p.dw = take((size_t)p.dw_way.splits * up(out, 32) * p.ld * 4);
    p.db = take((size_t)p.chunks * out * 4);
    p.bytes = at;
    return p;
}

// us of the gradients in one launch / in two or three, recorded and by calls (which wait for the host): 128 x 128 x 128 bf16 6.3 /
// 6.8 and 9.9 / 16, fp32 5.2 / 8.0 and 8.0 / 11.9; 128 x 512 x 128 fp32 9.0 / 8.0 and 8.0 / 11.8; 128 x 1024 x 128 bf16 11.1 /
// 6.9 and 11.2 / 16; 256 x 256 x 256 bf16 14.5 / 7.7 and 14.5 / 12.
bool small_fit(int B, int in, int out) {
    return B <= kSmallMost && out <= kSmallMost && in <= kSmallMostIn;
}

int blocks_for(size_t threads) { return (int)std::max<size_t>(1, std::min<size_t>((threads + 255) / 256, 148 * 8)); }

}  // namespace

void block8_wait_polls(int polls) { t_wait_polls = polls; }
unsigned block8_polls() { return t_wait_polls >= 0 ? (unsigned)t_wait_polls : kSpinLimit; }

int launch_fc8_fwd(int prec, const void *xq, const float *xs, const void *wq, const float *ws, const void *bias, void *y, int B, int in, int out, int y_f32, Launch s) {
    const int pitch = act8_pitch(in);
    if (rows_fit(B, in, out)) {
        const int nt = rows_columns(B), tiles = (out + kHalf - 1) / kHalf, x_tiles = (B + nt - 1) / nt, kw = nt <= 32 ? RowsStage<16>::kw : RowsStage<64>::kw;
        RowsArgs g{};
        g.B = B; g.out = out; g.tiles = tiles; g.steps = (in + kw - 1) / kw; g.splits = rows_splits(nt, tiles * x_tiles, in);
        g.tail = (in - (g.steps - 1) * kw + 31) / 32;
        g.row_scale = xs; g.col_scale = ws; g.bias = bias; g.bias_bf16 = prec == P_BF16; g.y = y; g.out_bf16 = prec == P_BF16 && !y_f32;
        g.vec = out % 4 == 0 && (reinterpret_cast<uintptr_t>(y) & (g.out_bf16 ? 7 : 15)) == 0;
        g.polls = block8_polls();
        CUtensorMap mw, mx;
        if (!box_map(CU_TENSOR_MAP_DATA_TYPE_UINT8, 1, wq, out, in, pitch, kHalf, &mw) || !box_map(CU_TENSOR_MAP_DATA_TYPE_UINT8, 1, xq, B, in, pitch, nt, &mx)) return -1;
        switch (nt) {
        case 16: return rows_launch<16>(mw, mx, g, tiles * x_tiles, s);
        case 32: return rows_launch<32>(mw, mx, g, tiles * x_tiles, s);
        case 64: return rows_launch<64>(mw, mx, g, tiles * x_tiles, s);
        default: return rows_launch<128>(mw, mx, g, tiles * x_tiles, s);
        }
    }
    MmArgs g{};
    g.M = B; g.N = out; g.n_seg = 1; g.splits = 1; g.width = mm_width(B, out, 1, kPairs);
    g.row_scale = xs; g.col_scale = ws; g.bias = bias; g.bias_bf16 = prec == P_BF16;
    mm_out(g, y, prec == P_BF16 && !y_f32, out);
    MmLaunch<kForward> mm;
    return mm.add(Operand{xq, B, in, (size_t)pitch}, Operand{wq, out, in, (size_t)pitch}, g, in, in, true) ? mm.run<false>(s) : -1;
}

size_t fc8_workspace_bytes(int prec, int B, int in, int out) { return bwd_plan(prec, B, in, out).bytes; }

template <typename T, typename TW>
static int small_bwd(const void *dy, const void *xq, const float *xs, const void *wq, const float *ws, void *dx, void *dW, float *db, int B, int in, int out, const Launch &s) {
    SmallArgs g{dy, (const int8_t *)xq, (const int8_t *)wq, xs, ws, dx, dW, db, B, in, out, act8_pitch(in)};
    const int tiles_n = (in + kSmallN - 1) / kSmallN;
    g.dx_tiles = dx ? (B + kSmallM - 1) / kSmallM * tiles_n : 0;
    g.dw_tiles = dW ? (out + kSmallM - 1) / kSmallM * tiles_n : 0;
    launch_k(fc8_small_bwd_kernel<T, TW>, g.dx_tiles + g.dw_tiles + (db ? (out + 63) / 64 : 0), 256, 0, s, g);
    return 1;
}

int launch_fc8_bwd(int prec, const void *dy, const void *xq, const float *xs, const void *wq, const float *ws, void *dx, void *dW, float *db, void *ws_mem, int B, int in, int out,
                   int dw_f32, Launch s) {
    if (small_fit(B, in, out)) {
        if (prec == P_F32) return small_bwd<float, float>(dy, xq, xs, wq, ws, dx, dW, db, B, in, out, s);
        return dw_f32 ? small_bwd<bf16, float>(dy, xq, xs, wq, ws, dx, dW, db, B, in, out, s) : small_bwd<bf16, bf16>(dy, xq, xs, wq, ws, dx, dW, db, B, in, out, s);
    }
    const BwdPlan p = bwd_plan(prec, B, in, out);
    uint8_t *base = (uint8_t *)ws_mem;
    const int pitch = act8_pitch(in);
    const bool f32 = prec == P_F32, aligned = (reinterpret_cast<uintptr_t>(dy) & 15) == 0, copy = f32 || out % 8 != 0 || !aligned;
    PrepArgs prep{};
    int n = 0, blocks = 0;
    auto codes = [&](int k, const void *q, const float *scale, size_t at, int rows) {
        prep.codes[k] = CodesJob{(const int8_t *)q, f32 ? nullptr : scale, (bf16 *)(base + at), rows, pitch, p.plane_in, blocks_for((size_t)rows * (pitch / 16))};
        blocks += prep.codes[k].blocks;
    };
    if (dx) codes(0, wq, ws, p.w, out);
    if (dW) codes(1, xq, xs, p.x, B);
    if (copy && (dx || dW)) {
        auto to = [&](int k, bool wanted) { return wanted ? (bf16 *)(base + p.dy[k]) : nullptr; };
        prep.terms = TermsJob{dy, to(0, !f32), to(0, f32 && dx), to(1, f32 && dW), xs, ws, B, out, p.plane_out, p.planes,
                              blocks_for((size_t)B * ((p.plane_out + kTermCols - 1) / kTermCols) * 32)};
        blocks += prep.terms.blocks;
    }
    if (db) {
        prep.sums = SumsJob{dy, p.chunks > 1 ? (float *)(base + p.db) : db, B, out, p.chunk, p.chunks * ((out + 63) / 64), out % (f32 ? 4 : 8) == 0 && aligned};
        blocks += prep.sums.blocks;
    }
    if (f32) launch_k(fc8_prep_kernel<float>, blocks, 256, 0, s, prep); else launch_k(fc8_prep_kernel<bf16>, blocks, 256, 0, s, prep);
    ++n;
    const int dy_cols = copy ? (f32 ? p.planes * p.plane_out : out) : out;
    const size_t dy_ld = copy ? (size_t)p.planes * p.plane_out : (size_t)out;
    auto operand = [&](int k) { return Operand{copy ? base + p.dy[f32 ? k : 0] : dy, B, dy_cols, dy_ld}; };
    auto segments = [&](MmArgs &g) {  // the smallest terms first
        g.n_seg = p.planes;
        for (int i = 0; i < p.planes; ++i) g.a_off[i] = (p.planes - 1 - i) * p.plane_out;
    };
    JoinArgs join{};
    int join_blocks = 0, joins = 0;
    auto joined = [&](const MmArgs &g, size_t part, void *to, bool is_bf16) {
        const size_t total = (size_t)g.M * (g.ld / 4);
        join.job[joins++] = JoinJob{(const float *)(base + part), to, g.out_split, total, g.splits, g.ld, in, is_bf16, in % 4 == 0 && (reinterpret_cast<uintptr_t>(to) & (is_bf16 ? 7 : 15)) == 0,
                                    blocks_for(total)};
        join_blocks += join.job[joins - 1].blocks;
    };
    const bool dw_bf16 = !f32 && !dw_f32;
    const bool together = dx && dW && mm_together(p.dx_way, p.dw_way), dw_first = together && p.dw_way.each > p.dx_way.each;
    MmLaunch<kGrad> mm;
    bool promote = false;
    auto product = [&](bool a_mn, const Operand &a, const Operand &b, int M, int K, const MmWay &way, size_t part, void *to, bool is_bf16, bool last) {
        MmArgs g{};
        g.M = M; g.N = in; g.splits = way.splits; g.width = together ? way.width : mm_width(M, in, way.splits, kPairs); g.a_mn = a_mn;
        segments(g);
        if (g.splits > 1) mm_out(g, base + part, false, p.ld); else mm_out(g, to, is_bf16, in);
        const int most = is_bf16 ? kPieceOut : kPieceF32;
        const bool cut = (long)K * g.n_seg / g.splits > most;  // by the product's own sizes, whatever it shares the launch with
        promote = promote || cut;
        if (g.splits > 1) joined(g, part, to, is_bf16);
        return mm.add(a, b, g, K, cut ? most : kWhole, last);
    };
    auto run = [&]() {
        const int r = promote ? mm.run<true>(s) : mm.run<false>(s);
        mm = MmLaunch<kGrad>();
        promote = false;
        return r;
    };
    for (int k = 0; k < 2; ++k) {
        const bool of_x = (k == 0) != dw_first, last = k == 1 || !together;
        if (!(of_x ? dx : dW)) continue;
        if (!(of_x ? product(false, operand(0), Operand{base + p.w, out, in, (size_t)p.plane_in}, B, out, p.dx_way, p.dx, dx, !f32, last)
                   : product(true, operand(1), Operand{base + p.x, B, in, (size_t)p.plane_in}, out, B, p.dw_way, p.dw, dW, dw_bf16, last)))
            return -1;
        if (!last) continue;
        const int r = run();
        if (r < 0) return r;
        n += r;
    }
    if (db && p.chunks > 1) {
        join.sums = JoinSums{(const float *)(base + p.db), db, p.chunks, out};
        join_blocks += (out + 31) / 32;
    }
    if (join_blocks) {
        launch_k(fc8_join_kernel, join_blocks, 256, 0, s, join);
        ++n;
    }
    return n;
}

}  // namespace ddg

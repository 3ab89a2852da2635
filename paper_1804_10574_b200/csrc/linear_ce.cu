// Vocabulary projection with softmax cross entropy, in pieces of the vocabulary: the logits z = x W^T + b ([B][V], far
// larger than x and W for a large vocabulary V) exist only in tensor memory, one 256 x 256 tile at a time.
//
//   forward    z_nv = sum_d x_nd W_vd + b_v;  lse_n = log sum_v exp z_nv;  l_n = lse_n - z_n,y_n
//              one GEMM whose epilogue keeps, per row and 128 columns, the maximum and the sum of exp(z - maximum); a
//              small kernel joins the pieces.
//   backward   dz_nv = (exp(z_nv - lse_n) - [v = y_n]) g_n, one chunk of the vocabulary at a time:
//                1. z again, dz of the chunk to the workspace (bf16),
//                2. dx += dz W_chunk       (fp32 partial sums, one per split of the chunk's columns)
//                3. dW_chunk = dz^T x
//              and at the end dx = scale * (sum of its partials).
//
// All products run on one tcgen05 kernel (a few rows and small heads have kernels of their own, linear_ce_rows.cuh,
// linear_ce_rows32.cuh and linear_ce_head.cuh).  What bounds it: 2NVD (forward) and 6NVD (backward) multiply-adds on the tensor cores.  Two CTAs of
// a cluster work on one tile of 256 x 256 or 256 x 512 (cta_group::2): each loads half of A and half of B by TMA, three
// stages of 64 KB or four of 48 KB.  The 512 TMEM columns are two accumulators of 256: successive tiles of the narrow
// form, or the halves of a wide tile; what the epilogue warps do with one (128 columns of a row per thread) runs under the
// products of the other.  Measured (bf16, TFLOP/s of the products that are needed, z computed twice counted twice):
//   8192 x 4096 x 65536   forward 1660, backward 1580 in short runs; 1460 and 1360 for seconds on end, under the power cap
//   4096 x 1024 x 32000   forward 1450, backward 1400; 1390 and 1240
//
// The accumulator truncates, so that a chain of many steps of 16 products ends too small.  Products of both signs: 2048 of
// them are off by 3e-7 at most.  Products of one sign, relative to their sum: 1024 of them 6.6e-7, 2048 2.6e-6, 2^20 2.3e-3,
// 2^22 2.2e-2, 2^24 a tenth.  Where a result stays in 32 bits, chains are cut after 1024 products (fewer for a few rows), for
// fp32 tensors after every block of 128 K values, and the pieces added in registers, rounded to nearest: lse of 4096 x 2048 x
// 32000 is 3.5e-6 off 64 bits, 7.6e-6 with chains of 2048, which take 1 to 5 % less between 1024 and 2048 columns and nothing
// less elsewhere.  Where the result is rounded to bf16 itself (dx, dW), they are cut after 65536 products (rows, or columns of
// a chunk): 1.5e-4 by proportion, a twentieth of that rounding.
//
// fp32 tensors are split into three bf16 terms each (x = h + m + l to 24 bits) and the products h h, h m, m h, m m, h l,
// l h are accumulated: what is left out is below 2^-24 of the value.  A block of K values goes through all six, smallest
// first, before the next block: the five small ones, 2^-8 of the result at most, lose nothing that shows, so that h h's
// eight steps are the chain (1111 x 520 x 10007: dx 2.1e-7 off 64 bits, the plain form 7.5e-7), and a block's terms are read
// from memory once and from the L2 after that (214 x 3816 x 16384, forward and backward: 868 -> 806 us against one product
// after the other over all of K).
#include <float.h>

#include <algorithm>

#include "cluster.cuh"
#include "common.cuh"
#include "conv_tc.h"
#include "lm_ops.h"
#include "tc_common.cuh"

namespace ddg {

namespace {

constexpr int kTile = 256;        // rows of a tile of the CTA pair, columns of an accumulator
constexpr int kHalf = 128;        // rows of A, and of B per accumulator, that one CTA of the pair loads
constexpr int kKBox = 64;         // K values of a box: 128 bytes of bf16, one swizzle row
// A stage, per CTA: 128 rows of A and 128 or 256 of B, 128 or 64 K values wide.  The thread that issues the products spends
// a few hundred cycles on a stage (two barriers, eight descriptors), which has to stay below the 1024 cycles that they
// take: with 64 K values the narrow tile kept the tensor cores 80 % busy (4096 x 1024 x 32000), with 128 91 %.
template <int NT> struct Stage {  // NT: columns of a tile
    static constexpr int kw = NT == kTile ? 2 * kKBox : kKBox;
    static constexpr int block = kHalf * kw * 2;  // one operand's 128 rows
    static constexpr int bytes = (1 + NT / kTile) * block;
    static constexpr int count = 192 * 1024 / bytes;
};
constexpr int kEpiWarps = 8;      // two per TMEM lane quarter, each half of an accumulator's columns
constexpr int kThreads = 64 + 32 * kEpiWarps;
constexpr int kStageRing = 192 * 1024;
constexpr int kOutBuf = 32 * kKBox * 2;  // an epilogue warp's 32 rows of 64 bf16 values on their way out
constexpr int kCeSmem = kStageRing + kEpiWarps * kOutBuf + 1024;
constexpr int kMaxSeg = 6;
// K values (times products) of a chain that need not be cut: for a 32-bit result of bf16 and of fp32 tensors, for a bf16 result
constexpr int kPieceBf16 = 1024, kPieceF32 = 256, kPieceOut = 65536;
constexpr float kLog2e = 1.4426950408889634f;

enum Mode { kLse, kDz, kPartial, kWeightGrad };

// What the workspace starts with.  A wait that runs out makes the results of its call NaN, all of them, and no other
// call's: the backward pass, whose first kernel clears `failed`, ends with a kernel that looks at it; the forward pass may
// have no kernel before the one that waits, so there every block leaves a word of its own, whatever stood there before.
constexpr int kMostBlocks = 160;  // of a kernel that waits
struct CeHeader {
    unsigned ticket;    // blocks of the joining kernel that are done
    float scale;        // factor on dx and dW: upstream gradient / counted rows
    int failed;         // backward: a wait of this call ran out
    int pad[93];
    int status[kMostBlocks];  // forward: a wait of this block ran out
};
static_assert(sizeof(CeHeader) == 1024, "the buffers behind the header stay aligned");

enum Out { kStore, kAdd, kFinal };

struct CeGemm {
    int M, N;                 // rows of A, rows of B (columns of the result)
    int K, kblocks, n_seg;    // K values and blocks of a segment; segments: pairs of bf16 terms
    int a_off[kMaxSeg], b_off[kMaxSeg];  // where a segment's term starts: in K (K-major operand) or in M / N
    int b_r0, b_k0;           // coordinates of B's first row and of its first K value
    int tiles_m, tiles_n, splits, group_m;
    int width;                // columns of a tile: at most NT, a multiple of 64, alike for all tiles of a launch
    int b_bytes;              // of B in a stage, per accumulator and CTA
    int piece;                // steps of the K range (K blocks times segments) of a chain (with PROMOTE)
    int tail;                 // steps of 16 in a segment's last K block
    CeHeader *head;
    // kLse, kDz
    const void *bias;         // nullable, at column 0 of this launch
    int bias_bf16;
    const int *labels;        // label of every row; columns are v0 + n
    int v0, V;
    float2 *part;             // kLse: [2 tiles_n][M] (maximum, sum)
    float *zlab;              // kLse: logit of the label
    const float *lse, *drow;  // kDz
    int planes, dz_plane;     // kDz: dz is [M][planes * dz_plane]
    float *db_part;           // kDz, nullable: [ceil(M / 32)][dz_plane]
    // kPartial (dx): fp32 sums [splits][M][ld] stored or added to, or, as kFinal, dx itself [M][N] from the product and
    // the sums so far (part_in, nullable).  kWeightGrad: [M][N].
    void *out;
    int out_kind, out_bf16, out_tma, ld;  // out_tma: bf16 that a tensor map can write
    size_t out_split;
    const float *part_in;
    unsigned polls;           // of a bounded wait
    int pairs;                // CTA pairs of the launch
};

// Hands an accumulator back.  What it orders are the tcgen05 loads before the fence, not memory: a releasing arrival would
// wait for the stores of the tile before (gradient of the logits, 4096 x 512 x 16384: 94 us with it, 89 us without).
__device__ __forceinline__ void mbar_arrive_remote(uint32_t cluster_addr) {
    asm volatile("mbarrier.arrive.relaxed.cluster.shared::cluster.b64 _, [%0];" ::"r"(cluster_addr) : "memory");
}
// one half of a stage: lands in this CTA's shared memory, counts on the barrier of the pair's first CTA
__device__ __forceinline__ void tma_load_pair(uint32_t dst, const CUtensorMap *map, uint32_t cluster_bar, int c0, int c1) {
    asm volatile(
        "cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4}], [%2];"
        ::"r"(dst), "l"(map), "r"(cluster_bar), "r"(c0), "r"(c1)
        : "memory");
}
__device__ __forceinline__ void mma_pair(uint32_t d_tmem, uint64_t adesc, uint64_t bdesc, uint32_t idesc, uint32_t accumulate) {
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n\t}"
        ::"r"(d_tmem), "l"(adesc), "l"(bdesc), "r"(idesc), "r"(accumulate)
        : "memory");
}
__device__ __forceinline__ bool elect_one() {
    uint32_t ok;
    asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(ok));
    return ok != 0;
}
// arrives on the barrier at this offset in both CTAs when the MMAs issued so far are done
__device__ __forceinline__ void commit_pair(uint32_t bar) {
    asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;"
                 ::"r"(bar), "h"((uint16_t)3) : "memory");
}
// Waits for work that is known to be in flight, which ends by itself: the limit is there for broken hardware alone.
__device__ __forceinline__ void mbar_drain(uint32_t bar, uint32_t parity) {
    for (unsigned i = 0; i < kSpinLimit; ++i) {
        if (mbar_try(bar, parity)) return;
        if (i > 4096) __nanosleep(64);
    }
}
constexpr uint32_t kGaveUp = 1u << 31;
__device__ __forceinline__ float exp2_approx(float v) { float r; asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(v)); return r; }

// Which tile a work item is: all tiles of a split, in bands of group_m tile rows that are walked column by column, so
// that the operands of the tiles in flight stay in the L2 (16 tile rows; 8 and 32 cost 2 to 5 % at 8192 x 4096 x 65536).
// Divisions by sizes known at launch only cost an issuing thread a hundred cycles each, in which the tensor cores run
// dry: the K range has none without splits, and the product of the two factors fits 32 bits (at most 2^21 x 148).
struct CeTile { int m, n; };
__device__ __forceinline__ int ce_split(const CeGemm &g, int item) { return g.splits == 1 ? 0 : item / (g.tiles_m * g.tiles_n); }
__device__ __forceinline__ void ce_range(const CeGemm &g, int split, int &kb0, int &kb1) {
    const int kb = g.kblocks * g.n_seg;
    kb0 = 0;
    kb1 = kb;
    if (g.splits > 1) {
        kb0 = (int)((unsigned)(kb * split) / (unsigned)g.splits);
        kb1 = (int)((unsigned)(kb * (split + 1)) / (unsigned)g.splits);
    }
}
// End of the chain that starts at step i of the K range (with PROMOTE): chains end where a K block's last product, h h, does.
__device__ __forceinline__ int ce_piece_end(const CeGemm &g, int i, int kb1) {
    return min(i + g.piece - (int)((unsigned)i % (unsigned)g.piece), kb1);
}
__device__ __forceinline__ CeTile ce_tile(const CeGemm &g, int item, int split) {
    unsigned r = (unsigned)(item - split * g.tiles_m * g.tiles_n);
    const unsigned band = r / (unsigned)(g.group_m * g.tiles_n);
    r -= band * g.group_m * g.tiles_n;
    const unsigned rows = min(g.group_m, g.tiles_m - (int)band * g.group_m), n = r / rows;
    return CeTile{(int)(band * g.group_m + r - n * rows), (int)n};
}

__device__ __forceinline__ uint32_t pack2(float a, float b) {
    const __nv_bfloat162 h = __floats2bfloat162_rn(a, b);
    return *reinterpret_cast<const uint32_t *>(&h);
}
__device__ __forceinline__ float bf16_round(float v) { return __bfloat162float(__float2bfloat16_rn(v)); }

__device__ __forceinline__ float load_bias(const void *bias, int is_bf16, int c) {
    return is_bf16 ? __bfloat162float(((const bf16 *)bias)[c]) : ((const float *)bias)[c];
}

// The sum over the warp's 32 rows of each of 32 columns: lane j ends with column j's.
__device__ __forceinline__ float column_sums(float (&v)[32], int lane) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            if (i < o) {
                const float keep = (lane & o) ? v[i + o] : v[i], send = (lane & o) ? v[i] : v[i + o];
                v[i] = keep + __shfl_xor_sync(0xffffffffu, send, o);
            }
        }
    }
    return v[0];
}

__device__ __forceinline__ void red_add4(float *p, float a, float b, float c, float d) {
    asm volatile("red.global.add.v4.f32 [%0], {%1, %2, %3, %4};" ::"l"(p), "f"(a), "f"(b), "f"(c), "f"(d) : "memory");
}

// 64 columns of the warp's 32 rows as bf16 to (x, y) of a matrix, through shared memory: whole 128-byte lines leave by
// TMA, and rows and columns past the matrix are clipped.  (Gradient of the logits, 4096 x 512 x 16384: 62 us; with stores
// of 64 bytes a thread, straight from registers, 89 us.)
__device__ __forceinline__ void store_box(const CUtensorMap *map, uint32_t buf, int lane, int x, int y, const float *v) {
    if (lane == 0) asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory");  // the box before has been read
    __syncwarp();
#pragma unroll
    for (int j = 0; j < 8; ++j)  // the 128-byte swizzle of the map
        asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(buf + lane * 128 + ((j ^ (lane & 7)) << 4)), "r"(pack2(v[8 * j], v[8 * j + 1])),
                     "r"(pack2(v[8 * j + 2], v[8 * j + 3])), "r"(pack2(v[8 * j + 4], v[8 * j + 5])), "r"(pack2(v[8 * j + 6], v[8 * j + 7]))
                     : "memory");
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    __syncwarp();
    if (lane == 0) {
        asm volatile("cp.async.bulk.tensor.2d.global.shared::cta.bulk_group [%0, {%2, %3}], [%1];" ::"l"(map), "r"(buf), "r"(x), "r"(y) : "memory");
        asm volatile("cp.async.bulk.commit_group;" ::: "memory");
    }
}

// The same for matrices that a tensor map cannot write (rows off 16-byte boundaries, fp32): rows row0 .. of a [rows][n]
// matrix, columns col .. col + 63 as far as there are; the lanes write neighbouring values of a row.  (7244 x 3955 x 223,
// forward and backward: 230 us; with a row per lane, two bytes at a time, here and in the copies, 499 us.)
template <bool BF16>
__device__ __forceinline__ void store_rows(void *out, uint32_t buf, int lane, int row0, int rows, int col, int n, const float *v) {
    const int last = min(32, rows - row0);
#pragma unroll
    for (int half = 0; half < (BF16 ? 1 : 2); ++half) {  // 128 bytes of a row at a time
        __syncwarp();  // what stood there has been read
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const float *f = v + (BF16 ? 8 * j : 32 * half + 4 * j);
            asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(buf + lane * 128 + ((j ^ (lane & 7)) << 4)), "r"(BF16 ? pack2(f[0], f[1]) : __float_as_uint(f[0])),
                         "r"(BF16 ? pack2(f[2], f[3]) : __float_as_uint(f[1])), "r"(BF16 ? pack2(f[BF16 ? 4 : 0], f[BF16 ? 5 : 0]) : __float_as_uint(f[2])),
                         "r"(BF16 ? pack2(f[BF16 ? 6 : 0], f[BF16 ? 7 : 0]) : __float_as_uint(f[3])) : "memory");
        }
        __syncwarp();
        const int c = col + 32 * half + lane;
#pragma unroll 4
        for (int r = 0; r < last; ++r) {
            const size_t at = (size_t)(row0 + r) * n + c;
            if (BF16) {
#pragma unroll
                for (int k = 0; k < 2; ++k) {  // columns lane and lane + 32
                    const int e = lane + 32 * k;
                    uint16_t w;
                    asm volatile("ld.shared.u16 %0, [%1];" : "=h"(w) : "r"(buf + r * 128 + (((e >> 3) ^ (r & 7)) << 4) + (e & 7) * 2));
                    if (c + 32 * k < n) reinterpret_cast<uint16_t *>(out)[at + 32 * k] = w;
                }
            } else {
                float w;
                asm volatile("ld.shared.f32 %0, [%1];" : "=f"(w) : "r"(buf + r * 128 + (((lane >> 2) ^ (r & 7)) << 4) + (lane & 3) * 4));
                if (c < n) reinterpret_cast<float *>(out)[at] = w;
            }
        }
    }
}

// What a thread knows of its row, and the softmax's running maximum and sum over the row's 128 columns.
struct CeRow {
    int split, row, label;  // label: column of this launch
    float lse, weight, top, sum;
};
template <int MODE> __device__ __forceinline__ CeRow ce_row(const CeGemm &g, int split, int row) {
    CeRow r{split, row, -1 - 2 * kTile, 0.f, 0.f, -INFINITY, 0.f};
    if (MODE != kWeightGrad && (MODE != kPartial || g.out_kind == kFinal) && row < g.M) {
        const int y = g.labels[row];
        const bool counted = y >= 0 && y < g.V;
        if (counted) r.label = y - g.v0;  // a label of another chunk meets no column
        if (MODE == kDz) r.lse = g.lse[row];
        r.weight = counted ? (MODE == kDz && g.drow ? g.drow[row] : 1.f) : 0.f;
    }
    return r;
}

// The bias of a warp's 128 columns, 32 per register and lane; columns past the vocabulary are masked later.
template <int MODE> __device__ __forceinline__ void ce_bias(const CeGemm &g, int col, int lane, float (&b)[4]) {
#pragma unroll
    for (int q = 0; q < 4; ++q) b[q] = (MODE == kLse || MODE == kDz) && g.bias ? load_bias(g.bias, g.bias_bf16, min(col + 32 * q + lane, g.N - 1)) : 0.f;
}

// What becomes of 64 columns of the warp's 32 rows: v at columns col .. of row r.row; b0 and b1: the columns' bias, a lane
// each, which the rows read from shared memory (s_bias, the warp's own).  (4096 x 64 x 18944, forward: 56 us; with the
// bias read from memory by every row, a column at a time, 83 us; without a bias 51 us.)
template <int MODE>
__device__ __forceinline__ void ce_finish(const CeGemm &g, const CUtensorMap *map_out, uint32_t buf, float *v, CeRow &r, int col, int lane, float *s_bias, float b0, float b1) {
    const bool live = r.row < g.M;
    if ((MODE == kLse || MODE == kDz) && g.bias) {
#pragma unroll
        for (int q = 0; q < 2; ++q) {
            __syncwarp();  // what stood there has been read
            s_bias[lane] = q ? b1 : b0;
            __syncwarp();
#pragma unroll
            for (int j = 0; j < 32; j += 4) {
                const float4 t = *reinterpret_cast<const float4 *>(s_bias + j);
                v[32 * q + j] += t.x; v[32 * q + j + 1] += t.y; v[32 * q + j + 2] += t.z; v[32 * q + j + 3] += t.w;
            }
        }
    }
    if (MODE == kLse) {
        if (col + kKBox > g.N) {
#pragma unroll
            for (int j = 0; j < kKBox; ++j)
                if (col + j >= g.N) v[j] = -INFINITY;
        }
        if (r.label >= col && r.label < col + kKBox) {
            float z = 0.f;
#pragma unroll
            for (int j = 0; j < kKBox; ++j)
                if (r.label == col + j) z = v[j];
            g.zlab[r.row] = z;
        }
        float m[4] = {r.top, v[1], v[2], v[3]};
#pragma unroll
        for (int j = 0; j < kKBox; ++j) m[j & 3] = fmaxf(m[j & 3], v[j]);
        const float top = fmaxf(fmaxf(m[0], m[1]), fmaxf(m[2], m[3]));
        const float ref = top == -INFINITY ? 0.f : top;  // nothing but -inf so far
        float s[4] = {r.sum * exp2_approx((r.top - ref) * kLog2e), 0.f, 0.f, 0.f};
#pragma unroll
        for (int j = 0; j < kKBox; ++j) s[j & 3] += exp2_approx((v[j] - ref) * kLog2e);
        r.top = top;
        r.sum = (s[0] + s[1]) + (s[2] + s[3]);
    } else if (MODE == kDz) {
#pragma unroll
        for (int j = 0; j < kKBox; ++j) v[j] = exp2_approx((v[j] - r.lse) * kLog2e);
        if (r.label >= col && r.label < col + kKBox) {
#pragma unroll
            for (int j = 0; j < kKBox; ++j)
                if (r.label == col + j) v[j] -= 1.f;
        }
        if (g.drow) {
#pragma unroll
            for (int j = 0; j < kKBox; ++j) v[j] *= r.weight;
        }
        // a row that does not count gives exact zeros whatever its logits are; so do columns past the vocabulary
        if (__any_sync(0xffffffffu, r.weight == 0.f)) {
#pragma unroll
            for (int j = 0; j < kKBox; ++j) v[j] = r.weight == 0.f ? 0.f : v[j];
        }
        if (col + kKBox > g.N) {
#pragma unroll
            for (int j = 0; j < kKBox; ++j)
                if (col + j >= g.N) v[j] = 0.f;
        }
        if (g.db_part) {  // rows that are not there hold zeros
            const int block = (r.row - lane) / 32;
#pragma unroll
            for (int c = 0; c < kKBox; c += 32) {
                float t[32];
#pragma unroll
                for (int j = 0; j < 32; ++j) t[j] = v[c + j];
                const float cs = column_sums(t, lane);
                if (block * 32 < g.M) g.db_part[(size_t)block * g.dz_plane + col + c + lane] = cs;
            }
        }
        if (r.row - lane < g.M) {
            for (int p = 0;;) {
                store_box(map_out, buf, lane, p * g.dz_plane + col, r.row - lane, v);
                if (++p == g.planes) break;
#pragma unroll
                for (int j = 0; j < kKBox; ++j) v[j] -= bf16_round(v[j]);
            }
        }
    } else if (r.row - lane < g.M) {
        if (MODE == kPartial && g.out_kind == kStore) {
            store_rows<false>((float *)g.out + r.split * g.out_split, buf, lane, r.row - lane, g.M, col, g.ld, v);
            return;
        }
        if (MODE == kPartial && g.out_kind == kAdd) {
            if (live) {
                float *dst = (float *)g.out + r.split * g.out_split + (size_t)r.row * g.ld + col;
#pragma unroll
                for (int j = 0; j < kKBox; j += 4)
                    if (col + j < g.ld) red_add4(dst + j, v[j], v[j + 1], v[j + 2], v[j + 3]);  // ld is a multiple of 4
            }
            return;
        }
        const float scale = g.head->scale;
        if (MODE == kPartial) {
            if (g.part_in && live) {
                const float *src = g.part_in + (size_t)r.row * g.ld + col;
#pragma unroll
                for (int j = 0; j < kKBox; j += 4)
                    if (col + j < g.ld) {
                        const float4 o = *reinterpret_cast<const float4 *>(src + j);
                        v[j] += o.x; v[j + 1] += o.y; v[j + 2] += o.z; v[j + 3] += o.w;
                    }
            }
#pragma unroll
            for (int j = 0; j < kKBox; ++j) v[j] = r.weight != 0.f ? v[j] * scale : 0.f;
        } else {
#pragma unroll
            for (int j = 0; j < kKBox; ++j) v[j] *= scale;
        }
        if (g.out_tma) store_box(map_out, buf, lane, col, r.row - lane, v);
        else if (g.out_bf16) store_rows<true>(g.out, buf, lane, r.row - lane, g.M, col, g.N, v);
        else store_rows<false>(g.out, buf, lane, r.row - lane, g.M, col, g.N, v);
    }
}

// A_MN / B_MN: the operand lies with M / N innermost (its rows are K values) instead of K.  NT: columns of a tile.
// PROMOTE (NT = 256): an accumulator holds at most g.piece steps, the epilogue adds the pieces.
template <int MODE, bool A_MN, bool B_MN, int NT, bool PROMOTE>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kThreads, 1)
ce_gemm_kernel(const __grid_constant__ CUtensorMap map_a, const __grid_constant__ CUtensorMap map_b,
               const __grid_constant__ CUtensorMap map_out, const __grid_constant__ CeGemm g) {
    static_assert(NT == kTile || (NT == 2 * kTile && !PROMOTE), "tiles are one or two accumulators wide");
    constexpr int kStages = Stage<NT>::count, kStageBytes = Stage<NT>::bytes, kBlockBytes = Stage<NT>::block, kw = Stage<NT>::kw, kHalves = NT / kTile;
    extern __shared__ uint8_t smem_raw[];
    __shared__ uint64_t full[kStages], empty[kStages], acc_full[2], acc_empty[2], drained;
    __shared__ uint32_t tmem_holder, s_peer;
    __shared__ int abort_flag;
    __shared__ float4 s_bias[MODE == kLse || MODE == kDz ? kEpiWarps : 1][8];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t rank = cluster_rank();
    const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u;
    const Waiter wt{&abort_flag, &abort_flag, g.polls};
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
    if (MODE == kLse && blockIdx.x == 0 && threadIdx.x == 0) g.head->ticket = 0;
    tc_fence_before();
    __syncthreads();
    cluster_sync();  // both CTAs' barriers are ready
    tc_fence_after();
    const uint32_t tmem = tmem_holder;
    const int n_items = g.tiles_m * g.tiles_n * g.splits;
    const int first = blockIdx.x >> 1, step = gridDim.x >> 1;
    // Copies into stage s of this CTA's halves of A and B: one step of the K range.
    auto load_step = [&](uint32_t s, int seg, int k, int m0, int n0) {
        if (rank == 0) mbar_expect_tx(smem_u32(&full[s]), 2u * (uint32_t)(kBlockBytes + kHalves * g.b_bytes));
        const uint32_t bar = map_rank(smem_u32(&full[s]), 0);
        const uint32_t a = base + s * kStageBytes;
        // K-major: a box is 64 K values of 128 rows.  MN-major: 64 rows of kw K values.
#pragma unroll
        for (int j = 0; j < (A_MN ? 2 : kw / kKBox); ++j) {
            if (A_MN) tma_load_pair(a + j * (kBlockBytes / 2), &map_a, bar, g.a_off[seg] + m0 + kKBox * j, k);
            else tma_load_pair(a + j * (kHalf * kKBox * 2), &map_a, bar, g.a_off[seg] + k + kKBox * j, m0);
        }
#pragma unroll
        for (int h = 0; h < kHalves; ++h) {
            const uint32_t b = a + (1 + h) * kBlockBytes;
            const int nn = n0 + h * kTile;
#pragma unroll
            for (int j = 0; j < (B_MN ? 2 : kw / kKBox); ++j) {
                if (B_MN && j * kKBox >= g.width / 2) break;
                if (B_MN) tma_load_pair(b + j * (kBlockBytes / 2), &map_b, bar, g.b_off[seg] + nn + kKBox * j, g.b_k0 + k);
                else tma_load_pair(b + j * (kHalf * kKBox * 2), &map_b, bar, g.b_off[seg] + k + kKBox * j, g.b_r0 + nn);
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
                const int split = ce_split(g, item);
                const CeTile t = ce_tile(g, item, split);
                int kb0, kb1;
                ce_range(g, split, kb0, kb1);
                const int m0 = t.m * kTile + (int)rank * kHalf, n0 = t.n * g.width + (int)rank * (NT == kTile ? g.width / 2 : kHalf);
                int kb = kb0 == 0 ? 0 : kb0 / g.n_seg, seg = kb0 - kb * g.n_seg;
                for (int i = kb0; i < kb1; ++i) {
                    if (!mbar_wait(smem_u32(&empty[s]), ph ^ 1u, wt, 51)) { ok = false; break; }
                    load_step(s, seg, kb * kw, m0, n0);
                    ++issued;
                    if (++seg == g.n_seg) { seg = 0; ++kb; }
                    if (++s == kStages) { s = 0; ph ^= 1u; }
                }
            }
        }
        __syncwarp();
    } else if (warp == 1) {
        if (rank == 0) {
            // Products, for both CTAs.  The tensor cores wait for this loop when a K block takes it longer to issue than to
            // multiply, so it is kept straight: the whole warp walks it and one elected lane issues; waits for an
            // accumulator and what follows its last K block stand outside (with them inside, under one lane,
            // 8192 x 4096 x 65536 took 3.56 ms instead of 2.92).
            issuer = elect_one();
            const uint32_t idesc = (1u << 4) | (1u << 7) | (1u << 10) | (A_MN ? 1u << 15 : 0u) | (B_MN ? 1u << 16 : 0u) |
                                   ((uint32_t)((NT == kTile ? g.width : kTile) >> 3) << 17) | ((uint32_t)(kTile >> 4) << 24);
            // K-major: 16 K values are 32 bytes of a swizzle row, the next 64 values 16 KB further.  MN-major: 16 rows of
            // 128 bytes; the next 64 of the 128 M / N values lie half a block further.
            const uint64_t ad0 = A_MN ? make_desc(base, 1024, 2u, kBlockBytes / 2) : make_desc(base, 1024, 2u);
            const uint64_t bd0 = B_MN ? make_desc(base + kBlockBytes, 1024, 2u, kBlockBytes / 2) : make_desc(base + kBlockBytes, 1024, 2u);
            auto multiply = [&](uint32_t s, int h, uint32_t acc, bool fresh, int steps) {
#pragma unroll
                for (int k = 0; k < kw / 16; ++k) {
                    if (k >= steps) break;
                    const uint32_t at = s * (kStageBytes >> 4), kk = (uint32_t)((k >> 2) * (kHalf * kKBox * 2 >> 4) + (k & 3) * 2);
                    mma_pair(tmem + acc * kTile, ad0 + (uint64_t)(at + (A_MN ? 128u * k : kk)),
                             bd0 + (uint64_t)(at + h * (kBlockBytes >> 4) + (B_MN ? 128u * k : kk)), idesc, !fresh || k > 0);
                }
            };
            bool ok = true;
            uint32_t s = 0, ph = 0, u = 0;  // stage, its parity, accumulators used so far
            for (int item = first; item < n_items && ok; item += step) {
                int kb0, kb1;
                const int split = ce_split(g, item);
                ce_range(g, split, kb0, kb1);
                const int short_from = (g.kblocks - 1) * g.n_seg;  // the last K block has g.tail steps of 16
                for (int i0 = kb0; i0 < kb1; u += kHalves) {
                    const int i1 = PROMOTE ? ce_piece_end(g, i0, kb1) : kb1;
                    // the first K block waits for the accumulators, one after the other
                    ok = mbar_wait(smem_u32(&full[s]), ph, wt, 53);
#pragma unroll
                    for (int h = 0; h < kHalves && ok; ++h) {
                        const uint32_t acc = (u + h) & 1u;
                        ok = mbar_wait(smem_u32(&acc_empty[acc]), (((u + h) >> 1) & 1u) ^ 1u, wt, 52);
                        tc_fence_after();
                        if (ok && issuer) multiply(s, h, acc, true, i0 >= short_from ? g.tail : kw / 16);
                    }
                    if (!ok) break;
                    if (issuer) commit_pair(smem_u32(&empty[s]));
                    if (++s == kStages) { s = 0; ph ^= 1u; }
                    for (int i = i0 + 1; i < i1; ++i) {
                        if (!mbar_wait(smem_u32(&full[s]), ph, wt, 53)) { ok = false; break; }
                        tc_fence_after();
                        if (issuer) {
                            if (i >= short_from) {
#pragma unroll
                                for (int h = 0; h < kHalves; ++h) multiply(s, h, (u + h) & 1u, false, g.tail);
                            } else {
#pragma unroll
                                for (int h = 0; h < kHalves; ++h) multiply(s, h, (u + h) & 1u, false, kw / 16);
                            }
                            commit_pair(smem_u32(&empty[s]));
                        }
                        if (++s == kStages) { s = 0; ph ^= 1u; }
                    }
                    if (!ok) break;
                    if (issuer) {
#pragma unroll
                        for (int h = 0; h < kHalves; ++h) commit_pair(smem_u32(&acc_full[(u + h) & 1u]));
                    }
                    i0 = i1;
                }
            }
        }
        __syncwarp();
    } else {
        const int quarter = warp & 3, half = (warp - 2) >> 2;
        uint32_t u = 0;
        bool ok = true;
        for (int item = first; item < n_items && ok; item += step) {
            const int split = ce_split(g, item);
            const CeTile t = ce_tile(g, item, split);
            const int row = t.m * kTile + (int)rank * kHalf + 32 * quarter + lane;
            int pieces = 1;
            if (PROMOTE) {
                int kb0, kb1;
                ce_range(g, split, kb0, kb1);
                pieces = 0;
                for (int i = kb0; i < kb1; i = ce_piece_end(g, i, kb1)) ++pieces;
            }
            float *const bias_s = reinterpret_cast<float *>(s_bias[MODE == kLse || MODE == kDz ? warp - 2 : 0]);
            const uint32_t buf = base + kStageRing + (uint32_t)(warp - 2) * kOutBuf;
#pragma unroll 1
            for (int h = 0; h < kHalves && ok; ++h) {
                const int first_col = h * kTile + half * kHalf, col0 = t.n * g.width + first_col, live = min(g.width - first_col, g.N - col0);
                CeRow r;
                float b[4];
                if (!PROMOTE) {  // loaded while the products run
                    r = ce_row<MODE>(g, split, row);
                    ce_bias<MODE>(g, col0, lane, b);
                }
                float v[PROMOTE ? kHalf : kKBox];
                if (PROMOTE) {
#pragma unroll
                    for (int j = 0; j < kHalf; ++j) v[PROMOTE ? j : 0] = 0.f;
                }
#pragma unroll 1
                for (int piece = 0; piece < pieces; ++piece, ++u) {
                    const uint32_t acc = u & 1u;
                    ok = __all_sync(0xffffffffu, mbar_wait(smem_u32(&acc_full[acc]), (u >> 1) & 1u, wt, 54));
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
                            if (c < live) ce_finish<MODE>(g, &map_out, buf, v, r, col0 + c, lane, bias_s, c == 0 ? b[0] : b[2], c == 0 ? b[1] : b[3]);
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
                if (!ok) break;
                if (PROMOTE) {
                    r = ce_row<MODE>(g, split, row);
                    ce_bias<MODE>(g, col0, lane, b);
#pragma unroll
                    for (int c = 0; c < kHalf; c += kKBox)
                        if (c < live) ce_finish<MODE>(g, &map_out, buf, v + c, r, col0 + c, lane, bias_s, b[c / 32], b[c / 32 + 1]);
                }
                if (MODE == kLse && row < g.M) g.part[(size_t)(2 * t.n + half) * g.M + row] = make_float2(r.top, r.sum);
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
        // step that only one of the CTAs has issued is completed by the other (any box will do), so that the barriers of all
        // steps complete: a step is at most kStages ahead of the products, so that no two of one stage are open.
        if (issuer) commit_pair(smem_u32(&drained));
        if (threadIdx.x == 0) mbar_drain(smem_u32(&drained), 0);
        __syncthreads();
        cluster_sync();
        if (threadIdx.x == 0) {
            const uint32_t peer = s_peer & ~kGaveUp, last = max(issued, peer);
            for (uint32_t i = issued; i < peer; ++i) load_step(i % kStages, 0, 0, 0, 0);
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
    if (threadIdx.x == 0) {
        if (MODE == kLse) g.head->status[blockIdx.x] = abort_flag;
        else if (abort_flag) g.head->failed = 1;
    }
    cluster_sync();
}

#include "linear_ce_rows.cuh"

#include "linear_ce_head.cuh"

#include "linear_ce_rows32.cuh"

// ---- joining the forward pass ----------------------------------------------------------------------------------------
// rows rows per block of 512 threads, the 512 / rows threads of a row share its pieces, eight loads in flight each.  The mean is taken by the block
// that finishes last, over the blocks' sums in index order.
constexpr int kJoin = 512;
__global__ void __launch_bounds__(kJoin) ce_join_kernel(const float2 *__restrict__ part, int n_part, const float *__restrict__ zlab, const int *__restrict__ labels,
                                                      float *__restrict__ loss, float *__restrict__ row_loss, float *__restrict__ lse_out,
                                                      double *__restrict__ sums, CeHeader *head, int n_status, int B, int V, int rows) {
    __shared__ float sm[kJoin], ss[kJoin];
    __shared__ double bl[32];
    __shared__ int bc[32], last;
    pdl_launch();
    pdl_wait();
    const int r = threadIdx.x & (rows - 1), t0 = threadIdx.x / rows, lanes = kJoin / rows;
    const int row = blockIdx.x * rows + r;
    const int status = (int)threadIdx.x < n_status ? head->status[threadIdx.x] : 0;
    float m = -INFINITY, s = 0.f;
    if (row < B) {
        for (int t = t0; t < n_part; t += 8 * lanes) {
            float2 q[8];
#pragma unroll
            for (int u = 0; u < 8; ++u) q[u] = t + u * lanes < n_part ? part[(size_t)(t + u * lanes) * B + row] : make_float2(-INFINITY, 0.f);
            float top = m;
#pragma unroll
            for (int u = 0; u < 8; ++u) top = fmaxf(top, q[u].x);
            const float ref = top == -INFINITY ? 0.f : top;
            s *= expf(m - ref);
#pragma unroll
            for (int u = 0; u < 8; ++u) s += q[u].y * expf(q[u].x - ref);
            m = top;
        }
    }
    sm[threadIdx.x] = m;
    ss[threadIdx.x] = s;
    const bool failed = __syncthreads_or(status) != 0;
    for (int o = lanes / 2; o > 0; o >>= 1) {
        if (t0 < o) {
            const int i = threadIdx.x, j = i + o * rows;
            const float top = fmaxf(sm[i], sm[j]), ref = top == -INFINITY ? 0.f : top;
            ss[i] = ss[i] * expf(sm[i] - ref) + ss[j] * expf(sm[j] - ref);
            sm[i] = top;
        }
        __syncthreads();
    }
    if (t0 == 0) {
        float l = 0.f;
        int counted = 0;
        if (row < B) {
            const int y = labels[row];
            float lse = logf(ss[r]) + sm[r];
            counted = y >= 0 && y < V;
            if (counted) l = lse - zlab[row];
            if (failed) l = lse = __int_as_float(0x7fffffff);
            if (lse_out) lse_out[row] = lse;
            if (row_loss) row_loss[row] = l;
        }
        bl[r] = (double)l;
        bc[r] = counted;
    }
    __syncthreads();
    if (threadIdx.x == 0) {
        double a = 0.0, c = 0.0;
        for (int i = 0; i < rows; ++i) { a += bl[i]; c += bc[i]; }
        sums[2 * blockIdx.x] = a;
        sums[2 * blockIdx.x + 1] = c;
        __threadfence();
        last = atomicAdd(&head->ticket, 1u) == gridDim.x - 1;
    }
    __syncthreads();
    if (last && loss) {
        __shared__ double fa[kJoin], fc[kJoin];
        __threadfence();
        double a = 0.0, c = 0.0;
        for (int i = threadIdx.x; i < (int)gridDim.x; i += kJoin) { a += __ldcg(sums + 2 * i); c += __ldcg(sums + 2 * i + 1); }
        fa[threadIdx.x] = a;
        fc[threadIdx.x] = c;
        __syncthreads();
        for (int o = kJoin / 2; o > 0; o >>= 1) {
            if ((int)threadIdx.x < o) { fa[threadIdx.x] += fa[threadIdx.x + o]; fc[threadIdx.x] += fc[threadIdx.x + o]; }
            __syncthreads();
        }
        if (threadIdx.x == 0) *loss = (float)(fa[0] / fmax(fc[0], 1.0));
    }
}

// ---- operands that TMA cannot read in place --------------------------------------------------------------------------
// dst [rows][planes * plane] bf16: term p of column c at p * plane + c, zero past `cols`.  labels (nullable): rows that do
// not count become zero, so that what stands in them (NaN among it) stays out of dW.  One launch copies up to two
// matrices (x and W), by `blocks` blocks each; when `count` is set one more block starts the backward pass's header.
// A job's rows from `again` on are its first ones once more; rows past the source's are zeros.
struct CePackJob { const void *src; bf16 *dst; const int *labels; int rows, blocks, src_rows, again; };
template <typename T>
__global__ void __launch_bounds__(256) ce_pack_kernel(const CePackJob job_x, const CePackJob job_w, int cols, int plane, int planes, int V, CeHeader *head, int count, int mean,
                                                      const int *__restrict__ labels_of_rows, int rows_of_labels, const float *__restrict__ dloss) {
    pdl_launch();
    pdl_wait();
    if (count && blockIdx.x == gridDim.x - 1) {
        __shared__ int part[256];
        int n = 0;
        if (mean) {
#pragma unroll 16
            for (int i = threadIdx.x; i < rows_of_labels; i += 256) n += labels_of_rows[i] >= 0 && labels_of_rows[i] < V;
        }
        part[threadIdx.x] = n;
        __syncthreads();
        for (int o = 128; o > 0; o >>= 1) {
            if ((int)threadIdx.x < o) part[threadIdx.x] += part[threadIdx.x + o];
            __syncthreads();
        }
        if (threadIdx.x == 0) {
            head->scale = mean ? (dloss ? *dloss : 1.f) / (float)max(part[0], 1) : 1.f;
            head->failed = 0;
        }
        return;
    }
    const bool second = (int)blockIdx.x >= job_x.blocks;
    const CePackJob &job = second ? job_w : job_x;
    const T *src = (const T *)job.src;
    const int *labels = job.labels;
    bf16 *dst = job.dst;
    const int first = blockIdx.x - (second ? job_x.blocks : 0);
    // an infinity or NaN stays in the first term alone (inf - inf would spread NaN into its row's others)
    auto rest = [](float v) {
        const float h = bf16_round(v);
        return isinf(h) || isnan(h) ? 0.f : v - h;
    };
    if (cols % (16 / (int)sizeof(T)) != 0 || (reinterpret_cast<uintptr_t>(src) & 15) != 0) {
        // rows off 16-byte boundaries: a warp per row, two neighbouring columns per lane
        const int lane = threadIdx.x & 31;
        for (int row = first * 8 + (threadIdx.x >> 5); row < job.rows; row += job.blocks * 8) {
            const int src_row = row >= job.again ? row - job.again : row;
            const int y = labels && src_row < job.src_rows ? labels[src_row] : 0;
            const bool live = src_row < job.src_rows && (!labels || (y >= 0 && y < V));
            const T *from = src + (size_t)src_row * cols;
            bf16 *to = dst + (size_t)row * planes * plane;
#pragma unroll 8
            for (int c = 2 * lane; c < plane; c += 64) {
                float a = live && c < cols ? to_f(from[c]) : 0.f, b = live && c + 1 < cols ? to_f(from[c + 1]) : 0.f;
                for (int p = 0; p < planes; ++p) {
                    *reinterpret_cast<uint32_t *>(to + (size_t)p * plane + c) = pack2(a, b);
                    a = rest(a);
                    b = rest(b);
                }
            }
        }
        return;
    }
    // eight columns per step; plane is a multiple of 8
    const size_t total = (size_t)job.rows * (plane / 8), stride = (size_t)job.blocks * 256;
    const unsigned per_row = plane / 8;
    for (size_t i = (size_t)first * 256 + threadIdx.x; i < total; i += stride) {
        const size_t row = total <= 0xffffffffu ? (unsigned)i / per_row : i / per_row;
        const int c = (int)(i - row * per_row) * 8;
        const size_t src_row = row >= (size_t)job.again ? row - job.again : row;
        float v[8];
        bool live = src_row < (size_t)job.src_rows;
        if (live && labels) { const int y = labels[src_row]; live = y >= 0 && y < V; }
        if (live && c < cols) {  // whole vectors: cols is a multiple of their length
            if (sizeof(T) == 2) {
                load_f<T, 8>(src + src_row * cols + c, v);
            } else {
                load_f<T, 4>(src + src_row * cols + c, reinterpret_cast<float(&)[4]>(v[0]));
                if (c + 4 < cols) {
                    load_f<T, 4>(src + src_row * cols + c + 4, reinterpret_cast<float(&)[4]>(v[4]));
                } else {
#pragma unroll
                    for (int j = 4; j < 8; ++j) v[j] = 0.f;
                }
            }
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] = 0.f;
        }
        for (int p = 0; p < planes; ++p) {
            *reinterpret_cast<uint4 *>(dst + row * planes * plane + (size_t)p * plane + c) =
                make_uint4(pack2(v[0], v[1]), pack2(v[2], v[3]), pack2(v[4], v[5]), pack2(v[6], v[7]));
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] = rest(v[j]);
        }
    }
}

// ---- ends of the backward pass ---------------------------------------------------------------------------------------
// db[c] = scale * sum over row blocks of part[block][c], for 32 columns per block of 256 threads: row blocks in index order
// per warp, warps in index order
struct CeDb { const float *part; float *db; int row_blocks, plane, cols; };
__device__ __forceinline__ void ce_db(const CeDb &g, int block, float scale) {
    __shared__ double fold[8][32];
    const int lane = threadIdx.x & 31, w = threadIdx.x >> 5, c = block * 32 + lane;
    double a = 0.0;
    if (c < g.cols) {
#pragma unroll 8
        for (int b = w; b < g.row_blocks; b += 8) a += (double)g.part[(size_t)b * g.plane + c];
    }
    fold[w][lane] = a;
    __syncthreads();
    if (w == 0 && c < g.cols) {
        for (int i = 1; i < 8; ++i) a += fold[i][lane];
        g.db[c] = (float)(a * (double)scale);
    }
}
// The results of a backward pass.
struct CeResults { void *dx, *dW; float *db; size_t n_dx, n_dw; int n_db, dx_bf16, dw_bf16; };
__device__ __forceinline__ void ce_fill_nan(void *p, size_t n, bool is_bf16) {
    for (size_t i = (size_t)blockIdx.x * blockDim.x + threadIdx.x; i < n; i += (size_t)gridDim.x * blockDim.x) {
        if (is_bf16) ((uint16_t *)p)[i] = 0x7fff; else ((uint32_t *)p)[i] = 0x7fffffffu;
    }
}
__device__ __forceinline__ bool ce_failed(const CeHeader *head, const CeResults &r) {
    if (!head->failed) return false;
    if (r.dx) ce_fill_nan(r.dx, r.n_dx, r.dx_bf16);
    if (r.dW) ce_fill_nan(r.dW, r.n_dw, r.dw_bf16);
    if (r.db) ce_fill_nan(r.db, r.n_db, false);
    return true;
}
// The end of a backward pass whose last kernel is not ce_dx_kernel.
__global__ void __launch_bounds__(256) ce_end_kernel(const CeHeader *head, const __grid_constant__ CeResults results) {
    pdl_launch();
    pdl_wait();
    ce_failed(head, results);
}
__global__ void __launch_bounds__(256) ce_db_kernel(const CeDb g, const CeHeader *head) {
    pdl_launch();
    pdl_wait();
    ce_db(g, blockIdx.x, head->scale);
}

// dx[n][c] = scale * sum_s part[s][n][c]; rows that do not count are zero.  The first db_blocks blocks fold db.  A block takes
// 256 / lanes groups of four columns at a time; `lanes` threads (1, or 8 where there are many splits and few columns)
// share a group's splits and are added in index order.
template <typename T>
__global__ void __launch_bounds__(256) ce_dx_kernel(const float *__restrict__ part, int splits, size_t split_stride, int ld, const int *__restrict__ labels, T *__restrict__ dx,
                                                    int B, int in, int V, int vec, int lanes, const CeHeader *head, const CeDb db, int db_blocks,
                                                    const __grid_constant__ CeResults results) {
    __shared__ float4 fold[256];
    pdl_launch();
    pdl_wait();
    if (ce_failed(head, results)) return;
    if ((int)blockIdx.x < db_blocks) {
        ce_db(db, blockIdx.x, head->scale);
        return;
    }
    const float scale = head->scale;
    const int groups = 256 / lanes, g = threadIdx.x & (groups - 1), lane = threadIdx.x / groups;
    const size_t total = (size_t)B * (ld / 4);
    for (size_t i0 = (size_t)(blockIdx.x - db_blocks) * groups; i0 < total; i0 += (size_t)(gridDim.x - db_blocks) * groups) {
        const size_t i = i0 + g, row = i / (ld / 4);
        const int c = (int)(i - row * (ld / 4)) * 4;
        float4 a = make_float4(0.f, 0.f, 0.f, 0.f);
        bool counted = false;
        if (i < total) {
            const int y = labels[row];
            counted = y >= 0 && y < V;
        }
        if (counted) {
#pragma unroll 8
            for (int s = lane; s < splits; s += lanes) {
                const float4 q = *reinterpret_cast<const float4 *>(part + s * split_stride + row * ld + c);
                a.x += q.x; a.y += q.y; a.z += q.z; a.w += q.w;
            }
        }
        if (lanes > 1) {
            __syncthreads();
            fold[threadIdx.x] = a;
            __syncthreads();
            if (lane != 0) continue;
            for (int l = 1; l < lanes; ++l) {
                const float4 q = fold[l * groups + g];
                a.x += q.x; a.y += q.y; a.z += q.z; a.w += q.w;
            }
        }
        if (i >= total) continue;
        float v[4] = {a.x * scale, a.y * scale, a.z * scale, a.w * scale};
        if (vec) {
            if (c < in) store_f<T, 4>(dx + row * in + c, v);
        } else {
#pragma unroll
            for (int j = 0; j < 4; ++j)
                if (c + j < in) dx[row * in + c + j] = from_f<T>(v[j]);
        }
    }
}

// ---- host side -------------------------------------------------------------------------------------------------------
int up(int v, int to) { return (v + to - 1) / to * to; }
size_t up256(size_t v) { return (v + 255) / 256 * 256; }

// Polls of a bounded wait, for the calls of this thread (negative: the default).
thread_local int t_wait_polls = -1;
unsigned wait_polls() { return t_wait_polls >= 0 ? (unsigned)t_wait_polls : kSpinLimit; }

int sm_count() {
    int dev = 0, n = 148;
    if (cudaGetDevice(&dev) == cudaSuccess) cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev);
    return n;
}

// A chunk of the vocabulary: dz of all rows for at most kDzBytes, at least one tile wide.  The chunk is written once and
// read twice; larger chunks mean fewer passes over the fp32 partial sums of dx.
constexpr size_t kDzBytes = (size_t)256 << 20;
constexpr int kPairs = 74;  // CTA pairs of the GPU: the splits of a plan (and with them the workspace) go by this number
constexpr double kWideCost = 0.97;  // time of a product in a 256 x 512 tile against a 256 x 256 one

// Columns of the tiles of M x N (times splits): at most 256, as many tiles as that takes, alike (520 columns: three of 192
// rather than 256, 256 and 8).  Where that leaves CTA pairs without work, narrower ones: half of a tile's loads, A's, stay.
// (105 x 1048 x 5130: forward 17.9 -> 17.0 us, backward 45.6 -> 39.5 us.)
int ce_width(int M, int N, int splits) {
    const long rows = (long)((M + kTile - 1) / kTile) * splits;
    int best = kTile;
    double least = 1e30;
    for (int most = kTile; most >= kKBox; most /= 2) {
        const int tiles = (N + most - 1) / most, width = ((N + tiles - 1) / tiles + kKBox - 1) / kKBox * kKBox;
        const double t = (double)((rows * tiles + kPairs - 1) / kPairs) * (0.5 + 0.5 * width / kTile);
        if (t < 0.98 * least) { least = t; best = width; }
        if (rows * tiles >= kPairs) break;
    }
    return best;
}
double ce_rounds(int M, int N, int nt, int splits);

struct CePlan {
    int planes, plane;       // terms of an element, columns of a term in a packed operand
    int dz_planes, chunk;    // terms of dz, columns of a chunk
    int dz_term, dz_cols;    // a few rows: columns between two terms of dz, columns of an entry's line
    int x_rows;              // of the copy of x
    int tiles_m, n_part;
    int splits, dx_ld;
    bool rows, rows32;       // a few rows: the kernels of linear_ce_rows.cuh, of linear_ce_rows32.cuh
    bool pack_x, pack_w;     // backward: x always, with the rows that do not count as zeros
    size_t part, zlab, sums, x, w, dz, db, dx, bytes;
};

// Few rows: columns of the MMA that hold the rows of x.
int rows_columns(int B) { return B <= 16 ? 16 : (B <= 32 ? 32 : 64); }
// Few rows: CTAs of the forward pass and of dz, at least one unit of the vocabulary each.
constexpr int kR32PerSm = 3;
int rows_grid(int out, int sms) { return std::min(std::min(sms, kMostBlocks), (out + kRowsUnit - 1) / kRowsUnit); }
// Few rows, dx: splits of the vocabulary, so that the tiles of 128 columns fill the SMs.  Seconds by the bytes of W and of
// the partial sums at 6 TB/s.
int rows_splits(int B, int in, int out, int ld) {
    const int tiles = (in + kHalf - 1) / kHalf, kb = (out + kRowsKw - 1) / kRowsKw, sms = 2 * kPairs;
    int best = 1;
    double least = 1e30;
    for (int n = 1; n <= std::max(1, std::min(sms, kb / 2)); ++n) {
        const double t = 2.0 * in * out / 6e12 * (double)((tiles * n + sms - 1) / sms) * sms / (tiles * n) + 8.0 * n * B * ld / 6e12;
        if (t < least) { least = t; best = n; }
    }
    return best;
}

CePlan ce_plan(int prec, int B, int in, int out, bool backward, bool dw_f32) {
    CePlan p{};
    p.planes = prec == P_F32 ? 3 : 1;
    // fp32: a stage never reaches into the next term.  bf16: rows that start on 128-byte lines
    p.plane = prec == P_F32 ? up(in, 2 * kKBox) : up(in, kKBox);
    // Rows of W that TMA can read but that do not start on 32-byte sectors cost every read of them a third more time (4096
    // rows, 32000 entries: 210 us at 1000 columns, 166 us at 1024); the copy costs the bytes of W twice and is paid for
    // by about 2000 rows (2001 x 1000 x 50021: 179 us without, about as much with it).
    p.pack_w = prec == P_F32 || in % 8 != 0 || (in % 16 != 0 && B >= 2048);
    p.rows32 = r32_fits(prec, B, in);
    if (p.rows32) p.pack_w = false;
    p.pack_x = p.pack_w || (backward && !p.rows32);
    // an fp32 dW of bf16 operands gets 16 bits of dz (two terms), as the fully connected layer's loss gradient does; a bf16
    // dW or dx is rounded to 8 bits itself and takes dz rounded once to bf16
    p.dz_planes = prec == P_F32 ? 3 : (dw_f32 ? 2 : 1);
    p.rows = prec == P_BF16 && B <= kRowsMax;
    if (p.rows) {  // up to 32 rows leave room for a second term in the line, see linear_ce_rows.cuh
        p.dz_term = rows_columns(B);
        if (p.dz_term < kRowsPitch) p.dz_planes = 2;
        p.dz_cols = p.dz_term < kRowsPitch ? kRowsPitch : p.dz_planes * kRowsPitch;
    }
    p.tiles_m = (B + kTile - 1) / kTile;
    p.n_part = p.rows || p.rows32 ? kMostBlocks * (p.rows32 ? kR32PerSm : 1) : 2 * ((out + ce_width(B, out, 1) - 1) / ce_width(B, out, 1));
    size_t at = sizeof(CeHeader);
    auto take = [&](size_t bytes) { const size_t r = at; at += up256(bytes); return r; };
    if (!backward) {
        p.part = take((size_t)p.n_part * B * sizeof(float2));
        p.zlab = take((size_t)B * 4);
        p.sums = take((size_t)B * 16);
    }
    p.x_rows = backward && p.rows && p.dz_term < kRowsPitch ? 2 * p.dz_term : B;  // dW = [both terms of dz]^T [x, x]: one product
    if (p.pack_x) p.x = take((size_t)p.x_rows * p.planes * p.plane * 2);
    if (p.pack_w) p.w = take((size_t)out * p.planes * p.plane * 2);
    if (backward && p.rows32) {
        p.chunk = out;
        p.dx_ld = up(in, 4);
        p.splits = std::max(1, std::min((r32_nb(B) == 16 ? 4 : 8) * kPairs / ((in + kR32Cols - 1) / kR32Cols), out / 64));  // two or four CTAs per SM
        p.dz = take((size_t)out * r32_nb(B) * 4);
        p.dx = take((size_t)p.splits * B * p.dx_ld * 4);
    } else if (backward && p.rows) {
        p.chunk = out;
        p.dx_ld = up(in, 4);
        p.splits = rows_splits(B, in, out, p.dx_ld);
        p.dz = take((size_t)out * p.dz_cols * 2);
        p.dx = take((size_t)p.splits * B * p.dx_ld * 4);
    } else if (backward) {
        const size_t fit = kDzBytes / ((size_t)B * p.dz_planes * 2) / kTile * kTile;
        p.chunk = (int)std::min<size_t>((size_t)up(out, kTile), std::max<size_t>(kTile, fit));
        p.dx_ld = up(in, 4);
        // dx: K is the chunk's columns.  It is split over CTA pairs where the tiles alone fill the GPU badly; each split
        // costs a write and a read of its partial sums.  Seconds by 1.4 PFLOP/s and 6 TB/s.
        const int kb = (int)std::min<long>(p.chunk, up(out, kKBox)) / kKBox * (prec == P_F32 ? 6 : 1);
        double best = 1e30;
        const int tiles = p.tiles_m * ((in + kTile - 1) / kTile), most = std::max(1, std::min(2 * kPairs / tiles, kb / 8));
        for (int i = 1; i <= 10; ++i) {  // 1 to 8, and one or two rounds of pairs
            const int n = std::min(most, i <= 8 ? i : (i - 8) * kPairs / tiles);
            if (n < 1) continue;
            const double rounds = prec == P_F32 ? ce_rounds(B, in, kTile, n) : std::min(ce_rounds(B, in, kTile, n), in > kTile ? ce_rounds(B, in, 2 * kTile, n) : 1e30);
            const double t = rounds * 2.0 * kTile * kTile * kKBox * kb * kPairs / 1.4e15 + (n > 1 ? 2e-6 + 8.0 * n * B * p.dx_ld / 6e12 : 0.0);
            if (t < best) { best = t; p.splits = n; }
        }
        p.dz = take((size_t)B * p.dz_planes * p.chunk * 2);
        p.db = take((size_t)((B + 31) / 32) * p.chunk * 4);
        if (p.splits > 1 || p.chunk < out) p.dx = take((size_t)p.splits * B * p.dx_ld * 4);
    }
    p.bytes = at;
    return p;
}

bool ce_map(const void *ptr, int rows, int cols, size_t ld, int box_rows, CUtensorMap *out) {
    PFN_cuTensorMapEncodeTiled_v12000 enc = tc_encode_fn();
    if (!enc) return false;
    cuuint64_t dims[2] = {(cuuint64_t)cols, (cuuint64_t)rows};
    cuuint64_t strides[1] = {(cuuint64_t)ld * 2};
    cuuint32_t box[2] = {(cuuint32_t)kKBox, (cuuint32_t)box_rows};
    cuuint32_t estr[2] = {1, 1};
    return enc(out, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, const_cast<void *>(ptr), dims, strides, box, estr,
               CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
               CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// An operand: a row-major bf16 matrix in memory.
struct CeOperand { const void *ptr; int rows, cols; };

template <int MODE, bool A_MN, bool B_MN, int NT, bool PROMOTE>
int ce_launch_as(const CeOperand &a, const CeOperand &b, const CeOperand &out, CeGemm &g, const Launch &s) {
    constexpr int kw = Stage<NT>::kw;
    g.kblocks = (g.K + kw - 1) / kw;
    g.tail = (g.K - (g.kblocks - 1) * kw + 15) / 16;
    g.piece = g.n_seg > 2 ? g.n_seg : std::max(1, kPieceBf16 / kw / g.n_seg) * g.n_seg;
    g.splits = std::max(1, std::min(g.splits, g.kblocks * g.n_seg));
    g.width = NT == kTile ? ce_width(g.M, g.N, g.splits) : NT;
    g.tiles_n = (g.N + g.width - 1) / g.width;
    const int b_rows = NT == kTile ? g.width / 2 : kHalf;  // per CTA and accumulator
    g.b_bytes = (B_MN ? (b_rows + kKBox - 1) / kKBox * kKBox : b_rows) * kw * 2;
    CUtensorMap ma, mb, mo{};
    if (out.ptr && !ce_map(out.ptr, out.rows, out.cols, out.cols, 32, &mo)) return -1;
    if (!ce_map(a.ptr, a.rows, a.cols, a.cols, A_MN ? kw : kHalf, &ma) || !ce_map(b.ptr, b.rows, b.cols, b.cols, B_MN ? kw : b_rows, &mb)) return -1;
    const long items = (long)g.tiles_m * g.tiles_n * g.splits;
    if (items > 0x7fffffff) return -1;
    static thread_local int ready_dev = -1;  // the attribute belongs to a device
    int dev = 0;
    cudaGetDevice(&dev);
    if (ready_dev != dev) {
        if (cudaFuncSetAttribute(ce_gemm_kernel<MODE, A_MN, B_MN, NT, PROMOTE>, cudaFuncAttributeMaxDynamicSharedMemorySize, kCeSmem) != cudaSuccess) return -1;
        ready_dev = dev;
    }
    g.polls = wait_polls();
    g.pairs = (int)std::min<long>(items, std::min(sm_count(), kMostBlocks) / 2);
    launch_k(ce_gemm_kernel<MODE, A_MN, B_MN, NT, PROMOTE>, 2 * g.pairs, kThreads, kCeSmem, s, ma, mb, mo, g);
    return 1;
}

// Rounds of the GPU's CTA pairs that the tiles (times splits) take, in units of one 256 x 256 tile of the whole K.
double ce_rounds(int M, int N, int nt, int splits) {
    const int width = nt == kTile ? ce_width(M, N, splits) : nt;
    const long items = (long)((M + kTile - 1) / kTile) * ((N + width - 1) / width) * splits;
    return (double)((items + kPairs - 1) / kPairs) * (nt == kTile ? 0.5 + 0.5 * width / kTile : 2 * kWideCost) / splits;
}
bool ce_wide(int M, int N, int splits) {
    return N > kTile && ce_rounds(M, N, 2 * kTile, splits) <= ce_rounds(M, N, kTile, splits);
}

// exact: the result stays in 32 bits (what chains are cut after: see the top of the file)
template <int MODE, bool A_MN, bool B_MN>
int ce_launch(const CeOperand &a, const CeOperand &b, const CeOperand &out, CeGemm &g, bool exact, const Launch &s) {
    g.tiles_m = (g.M + kTile - 1) / kTile;
    if (g.splits < 1) g.splits = 1;
    g.group_m = 16;
    const long chain = (long)g.K * g.n_seg / g.splits;
    if (chain > (!exact ? kPieceOut : (g.n_seg > 2 ? kPieceF32 : kPieceBf16))) return ce_launch_as<MODE, A_MN, B_MN, kTile, true>(a, b, out, g, s);
    // The softmax's epilogues are long, and a wide tile leaves no accumulator to multiply into meanwhile (forward pass,
    // 4096 x 1024 x 32000: 223 us wide, 200 us narrow, with stages alike); the other products' are short, a wide tile asks
    // a quarter less of the L2 (dW, 8192 x 4096 x 16384: 694 us wide, 720 us narrow), and the rounds decide.
    if constexpr (MODE == kPartial || MODE == kWeightGrad)
        if (ce_wide(g.M, g.N, g.splits)) return ce_launch_as<MODE, A_MN, B_MN, 2 * kTile, false>(a, b, out, g, s);
    return ce_launch_as<MODE, A_MN, B_MN, kTile, false>(a, b, out, g, s);
}

template <int MODE, int NT> int rows_launch_as(const CUtensorMap &w, const CUtensorMap &x, const CeRowsArgs &g, int grid, const Launch &s) {
    static thread_local int ready_dev = -1;
    int dev = 0;
    cudaGetDevice(&dev);
    if (ready_dev != dev) {
        if (cudaFuncSetAttribute(ce_rows_kernel<MODE, NT>, cudaFuncAttributeMaxDynamicSharedMemorySize, kRowsSmem) != cudaSuccess) return -1;
        ready_dev = dev;
    }
    launch_k(ce_rows_kernel<MODE, NT>, grid, kRowsThreads, kRowsSmem, s, w, x, g);
    return 1;
}
// the columns of the MMA: 16, 32 or 64 rows of x; for dx both terms of them where dz has two in a line
template <int MODE> int rows_launch(const CeOperand &w, const CeOperand &x, CeRowsArgs &g, const Launch &s) {
    g.polls = wait_polls();
    constexpr bool partial = MODE == kPartial;
    const int nt = std::min(kRowsPitch, (partial ? 2 : 1) * rows_columns(g.B));
    CUtensorMap mw, mx;
    if (!ce_map(w.ptr, w.rows, w.cols, w.cols, partial ? kRowsKw : kRowsUnit, &mw) || !ce_map(x.ptr, x.rows, x.cols, x.cols, partial ? kRowsKw : nt, &mx)) return -1;
    const int grid = partial ? std::min(g.tiles * g.splits, std::min(sm_count(), kMostBlocks)) : rows_grid(g.V, sm_count());
    if constexpr (!partial)
        if (nt == 16) return rows_launch_as<MODE, 16>(mw, mx, g, grid, s);
    return (nt == 32 ? rows_launch_as<MODE, 32>(mw, mx, g, grid, s) : rows_launch_as<MODE, 64>(mw, mx, g, grid, s));
}

// terms of A and of B that are multiplied, smallest products first
void ce_segments(CeGemm &g, int a_planes, int a_plane, int b_planes, int b_plane) {
    g.n_seg = 0;
    auto add = [&](int i, int j) {
        if (i < a_planes && j < b_planes) { g.a_off[g.n_seg] = i * a_plane; g.b_off[g.n_seg] = j * b_plane; ++g.n_seg; }
    };
    add(2, 0); add(0, 2); add(1, 1); add(1, 0); add(0, 1); add(0, 0);
}

// CTAs of the logits on an SM: two or three (registers) where x in shared memory leaves room for them
int r32_per_sm(int B, int in) { return std::max(1, std::min(r32_nb(B) == 16 ? 2 : kR32PerSm, (int)(kR32Smem / ((size_t)r32_nb(B) * r32_pitch(in) * 4)))); }
int r32_warps(int B, int in) { return r32_per_sm(B, in) > 1 ? 8 : kR32MostWarps; }
template <int MODE, int NB, int VEC> int r32_logits_as(const CeR32Args &g, int grid, const Launch &s) {
    static thread_local int ready_dev = -1;
    int dev = 0;
    cudaGetDevice(&dev);
    if (ready_dev != dev) {
        if (cudaFuncSetAttribute(ce_r32_logits_kernel<MODE, NB, VEC>, cudaFuncAttributeMaxDynamicSharedMemorySize, kR32Smem) != cudaSuccess) return -1;
        ready_dev = dev;
    }
    launch_k(ce_r32_logits_kernel<MODE, NB, VEC>, grid, 32 * r32_warps(g.B, g.D), (size_t)NB * r32_pitch(g.D) * sizeof(float), s, g);
    return 1;
}
template <int MODE> int r32_logits(const CeR32Args &g, int grid, const Launch &s) {
    const bool vec = g.D % 4 == 0 && (reinterpret_cast<uintptr_t>(g.W) & 15) == 0;
    switch (r32_nb(g.B)) {
    case 4: return vec ? r32_logits_as<MODE, 4, 4>(g, grid, s) : r32_logits_as<MODE, 4, 1>(g, grid, s);
    case 8: return vec ? r32_logits_as<MODE, 8, 4>(g, grid, s) : r32_logits_as<MODE, 8, 1>(g, grid, s);
    default: return vec ? r32_logits_as<MODE, 16, 4>(g, grid, s) : r32_logits_as<MODE, 16, 1>(g, grid, s);
    }
}
// CTAs of the logits: no more than give every warp a group of four entries
int r32_grid(int B, int in, int out) {
    return std::max(1, std::min(std::min(sm_count(), kMostBlocks) * r32_per_sm(B, in), (out + 31) / 32));
}
template <int NB> int r32_gradients(const CeR32Args &g, bool dx, const Launch &s) {
    const int slabs = (g.D + kR32Cols - 1) / kR32Cols;
    int n = 0;
    if (dx) {
        launch_k(ce_r32_dx_kernel<NB>, dim3(slabs, g.splits), kR32Threads, 0, s, g);
        ++n;
    }
    if (g.dW) {
        launch_k(ce_r32_dw_kernel<NB>, dim3(slabs, std::max(1, std::min(8 * kPairs / slabs, (g.V + 63) / 64))), kR32Threads, 0, s, g);
        ++n;
    }
    return n;
}

// Small heads: one launch per direction on the CUDA cores.  The eight CTAs of the forward pass take eight rows each at a time,
// which costs by the size of W; the other paths' two launches cost the same for all of these sizes, 10 us from 65 rows of bf16
// on (10 to 16 us up to 64).  One pass is faster everywhere (256 x 100: 10.1 us), two passes for a small W (64 x 100, 65 to 128 rows:
// 8.1 us; 128 x 10: 8.9; 32 x 300: 10.1 and 10.1; 256 x 100: 16.6 and 10.6), three never (64 x 100, 136 rows: 10.6 and 9.9).
// fp32, which the general path has to split: 256 x 64 x 100 14.3 us, 18 us.
bool head_fits(int prec, int B, int in, int out, bool backward) {
    const int most = backward || prec == P_F32 ? kHeadMaxB : (long)in * out <= 8192 ? 16 * kHeadRows : 8 * kHeadRows;
    return B <= most && in <= kHeadMaxD && head_smem(B, in, out) <= (size_t)kHeadSmem;
}
template <typename K> bool head_ready(K kernel, int &ready_dev) {
    int dev = 0;
    cudaGetDevice(&dev);
    if (ready_dev != dev) {
        if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kHeadSmem) != cudaSuccess) return false;
        ready_dev = dev;
    }
    return true;
}
template <typename T> int head_fwd(const CeHeadArgs &g, const Launch &s) {
    static thread_local int ready = -1;
    if (!head_ready(ce_head_fwd_kernel<T>, ready)) return -1;
    launch_k(ce_head_fwd_kernel<T>, 8, kHeadThreads, head_smem(g.B, g.D, g.V), s, g);
    return 1;
}
template <typename T> int head_bwd(const CeHeadArgs &g, const Launch &s) {
    static thread_local int ready = -1;
    if (!head_ready(ce_head_bwd_kernel<T>, ready)) return -1;
    const int row_ctas = g.dx ? (g.B + kHeadRows - 1) / kHeadRows : 0, slices = g.dW || g.db ? (g.V + kHeadRows - 1) / kHeadRows : 0;
    launch_k(ce_head_bwd_kernel<T>, row_ctas + slices, kHeadThreads, head_smem(g.B, g.D, g.V), s, g, row_ctas);
    return 1;
}

int grid_for(size_t threads) { return (int)std::max<size_t>(1, std::min<size_t>((threads + 255) / 256, 148 * 8)); }

// Copies x (nullable) and W (nullable) for TMA; backward: labels mask x's rows, and the scale is set.
int pack(int prec, const void *x, void *x_dst, const void *W, void *w_dst, const int *labels, const CePlan &p, int B, int in, int out, CeHeader *head, bool backward,
         bool mean, const float *dloss, const Launch &s) {
    CePackJob jx{x, (bf16 *)x_dst, backward ? labels : nullptr, p.x_rows, x ? grid_for((size_t)p.x_rows * (p.plane / 8)) : 0, B, p.x_rows > B ? p.dz_term : B};
    CePackJob jw{W, (bf16 *)w_dst, nullptr, out, W ? grid_for((size_t)out * (p.plane / 8)) : 0, out, out};
    const int grid = jx.blocks + jw.blocks + (backward ? 1 : 0);
    if (prec == P_BF16) launch_k(ce_pack_kernel<bf16>, grid, 256, 0, s, jx, jw, in, p.plane, p.planes, out, head, backward ? 1 : 0, mean ? 1 : 0, labels, B, dloss);
    else launch_k(ce_pack_kernel<float>, grid, 256, 0, s, jx, jw, in, p.plane, p.planes, out, head, backward ? 1 : 0, mean ? 1 : 0, labels, B, dloss);
    return 1;
}

int join_dx(int prec, const CePlan &p, uint8_t *base, const int *labels, const CeResults &results, int B, int in, int out, const CeDb &db, int db_blocks, const Launch &s) {
    void *dx = results.dx;
    const int lanes = p.splits >= 8 && (size_t)B * (p.dx_ld / 4) < 148 * 256 ? 8 : 1, grid = grid_for((size_t)B * (p.dx_ld / 4) * lanes) + db_blocks;
    const int vec = in % 4 == 0 && (reinterpret_cast<uintptr_t>(dx) & (4 * elem_size(prec) - 1)) == 0;
    const float *part = (const float *)(base + p.dx);
    const CeHeader *head = (const CeHeader *)base;
    if (prec == P_BF16)
        launch_k(ce_dx_kernel<bf16>, grid, 256, 0, s, part, p.splits, (size_t)B * p.dx_ld, p.dx_ld, labels, (bf16 *)dx, B, in, out, vec, lanes, head, db, db_blocks, results);
    else
        launch_k(ce_dx_kernel<float>, grid, 256, 0, s, part, p.splits, (size_t)B * p.dx_ld, p.dx_ld, labels, (float *)dx, B, in, out, vec, lanes, head, db, db_blocks, results);
    return 1;
}

}  // namespace

void linear_ce_wait_polls(int polls) { t_wait_polls = polls; }

bool linear_ce_in_place(int prec, int in) { return prec == P_BF16 && in % 8 == 0; }

size_t linear_ce_workspace_bytes(int prec, int B, int in, int out, int backward) {
    return std::max(ce_plan(prec, B, in, out, backward != 0, false).bytes, ce_plan(prec, B, in, out, backward != 0, true).bytes);
}

int launch_linear_ce_fwd(int prec, const void *x, const void *W, const void *bias, const int *labels, float *loss, float *row_loss, float *lse,
                         void *ws, int B, int in, int out, Launch s) {
    if (head_fits(prec, B, in, out, false)) {
        CeHeadArgs g{};
        g.x = x; g.W = W; g.bias = bias; g.labels = labels; g.loss = loss; g.row_loss = row_loss; g.lse_out = lse; g.B = B; g.D = in; g.V = out;
        return prec == P_BF16 ? head_fwd<bf16>(g, s) : head_fwd<float>(g, s);
    }
    const CePlan p = ce_plan(prec, B, in, out, false, false);
    uint8_t *base = (uint8_t *)ws;
    CeHeader *head = (CeHeader *)base;
    int n = 0;
    if (p.pack_w) {
        n += pack(prec, x, base + p.x, W, base + p.w, labels, p, B, in, out, head, false, false, nullptr, s);
        x = base + p.x;
        W = base + p.w;
    }
    const int cols = p.pack_w ? p.planes * p.plane : in;
    float2 *part = (float2 *)(base + p.part);
    float *zlab = (float *)(base + p.zlab);
    const CeOperand ox{x, B, cols}, ow{W, out, cols};
    int r, n_part = p.n_part, n_status;
    if (p.rows32) {
        CeR32Args g{};
        g.x = (const float *)x; g.W = (const float *)W; g.bias = (const float *)bias; g.labels = labels; g.head = head;
        g.part = part; g.zlab = zlab; g.B = B; g.D = in; g.V = out;
        n_part = r32_grid(B, in, out);
        n_status = 0;  // nothing waits
        r = r32_logits<kLse>(g, n_part, s);
    } else if (p.rows) {
        CeRowsArgs g{};
        g.B = B; g.D = in; g.V = out; g.head = head;
        g.bias = bias; g.bias_bf16 = 1; g.labels = labels; g.part = part; g.zlab = zlab;
        n_part = n_status = rows_grid(out, sm_count());
        r = rows_launch<kLse>(ow, ox, g, s);
    } else {
        CeGemm g{};
        g.M = B; g.N = out; g.K = in; g.head = head;
        ce_segments(g, p.planes, p.plane, p.planes, p.plane);
        g.bias = bias; g.bias_bf16 = prec == P_BF16; g.labels = labels; g.V = out;
        g.part = part; g.zlab = zlab;
        r = ce_launch<kLse, false, false>(ox, ow, CeOperand{}, g, true, s);
        n_status = 2 * g.pairs;
    }
    if (r < 0) return r;
    int rows = 1;  // of a block: as many blocks as SMs before rows share one
    while (rows < 32 && rows * 2 * kPairs < B) rows *= 2;
    launch_k(ce_join_kernel, (B + rows - 1) / rows, kJoin, 0, s, (const float2 *)part, n_part, (const float *)zlab, labels, loss, row_loss, lse,
             (double *)(base + p.sums), head, n_status, B, out, rows);
    return n + r + 1;
}

int launch_linear_ce_bwd(int prec, const void *x, const void *W, const void *bias, const int *labels, const float *lse, const float *dloss,
                         const float *drow, void *dx, void *dW, float *db, void *ws, int B, int in, int out, int dw_f32, Launch s) {
    if (head_fits(prec, B, in, out, true) && dx != x) {  // its CTAs read x while others write dx
        CeHeadArgs g{};
        g.x = x; g.W = W; g.bias = bias; g.labels = labels; g.lse = lse; g.dloss = dloss; g.drow = drow; g.dx = dx; g.dW = dW; g.db = db;
        g.B = B; g.D = in; g.V = out; g.dw_f32 = dw_f32;
        return prec == P_BF16 ? head_bwd<bf16>(g, s) : head_bwd<float>(g, s);
    }
    const CePlan p = ce_plan(prec, B, in, out, true, dw_f32 != 0);
    uint8_t *base = (uint8_t *)ws;
    CeHeader *head = (CeHeader *)base;
    const CeResults results{dx, dW, db, (size_t)B * in, (size_t)out * in, out, prec == P_BF16, prec == P_BF16 && !dw_f32};
    if (p.rows32) {
        CeR32Args g{};
        g.x = (const float *)x; g.W = (const float *)W; g.bias = (const float *)bias; g.labels = labels; g.head = head;
        g.lse = lse; g.dloss = dloss; g.drow = drow; g.dz = (float *)(base + p.dz); g.db = db; g.dW = (float *)dW;
        g.dx_part = (float *)(base + p.dx); g.dx_split = (size_t)B * p.dx_ld; g.B = B; g.D = in; g.V = out; g.ld = p.dx_ld; g.splits = p.splits;
        const int r = r32_logits<kDz>(g, r32_grid(B, in, out), s);
        if (r < 0) return r;
        const int nb = r32_nb(B), k = r + (nb == 4 ? r32_gradients<4>(g, dx, s) : (nb == 8 ? r32_gradients<8>(g, dx, s) : r32_gradients<16>(g, dx, s)));
        return dx ? k + join_dx(prec, p, base, labels, results, B, in, out, CeDb{}, 0, s) : k;
    }
    int n = pack(prec, x, base + p.x, p.pack_w ? W : nullptr, base + p.w, labels, p, B, in, out, head, true, drow == nullptr, dloss, s);
    const void *xp = base + p.x;
    if (p.pack_w) W = base + p.w;
    const int x_cols = p.planes * p.plane, w_cols = p.pack_w ? p.planes * p.plane : in;
    const int dz_cols = p.dz_planes * p.chunk;
    bf16 *dz = (bf16 *)(base + p.dz);
    const CeOperand ox{xp, B, x_cols}, ow{W, out, w_cols}, oz{dz, B, dz_cols};
    const int es = prec == P_BF16 ? 2 : 4;
    const bool out_bf16 = prec == P_BF16 && !dw_f32;
    // dW for the vocabulary entries [v0, v0 + cols), from dz with entries innermost (general) or rows of x (few rows)
    auto weight_gradient = [&](int v0, int cols) {
        const int oe = out_bf16 ? 2 : 4;
        CeGemm g{};
        g.M = cols; g.N = in; g.head = head;
        g.out = (uint8_t *)dW + (size_t)v0 * in * oe; g.out_bf16 = out_bf16;
        g.out_tma = out_bf16 && in % 8 == 0 && (reinterpret_cast<uintptr_t>(dW) & 15) == 0;
        const CeOperand o = g.out_tma ? CeOperand{g.out, cols, in} : CeOperand{};
        if (p.rows) {
            const bool both = p.x_rows > B;
            g.K = both ? p.x_rows : kRowsPitch;
            ce_segments(g, both ? 1 : p.dz_planes, kRowsPitch, 1, 0);
            return ce_launch<kWeightGrad, false, true>(CeOperand{dz, out, p.dz_cols}, CeOperand{xp, p.x_rows, x_cols}, o, g, !out_bf16, s);
        }
        g.K = B;
        ce_segments(g, p.dz_planes, p.chunk, p.planes, p.plane);
        return ce_launch<kWeightGrad, true, true>(oz, ox, o, g, !out_bf16, s);
    };
    const bool dx_direct = !p.rows && p.splits == 1;  // the last chunk's product writes dx itself
    const bool db_last = db && dx && !p.rows && !dx_direct && p.chunk >= out;  // db is folded beside dx's partial sums
    const CeDb db_all{(const float *)(base + p.db), db, (B + 31) / 32, p.chunk, out};
    if (p.rows) {
        CeRowsArgs g{};
        g.B = B; g.D = in; g.V = out; g.head = head;
        g.bias = bias; g.bias_bf16 = 1; g.labels = labels; g.lse = lse; g.drow = drow;
        g.dz = dz; g.db = db; g.planes = p.dz_planes;
        int r = rows_launch<kDz>(ow, ox, g, s);
        if (r < 0) return r;
        n += r;
        if (dx) {
            g.tiles = (in + kHalf - 1) / kHalf; g.splits = p.splits;
            g.dx_part = (float *)(base + p.dx); g.dx_split = (size_t)B * p.dx_ld; g.ld = p.dx_ld;
            if ((r = rows_launch<kPartial>(ow, CeOperand{dz, out, p.dz_cols}, g, s)) < 0) return r;
            n += r;
        }
        if (dW) {
            if ((r = weight_gradient(0, out)) < 0) return r;
            n += r;
        }
    } else
    for (int v0 = 0; v0 < out; v0 += p.chunk) {
        const int cols = std::min(p.chunk, out - v0);
        {
            CeGemm g{};
            g.M = B; g.N = cols; g.K = in; g.head = head; g.b_r0 = v0;
            ce_segments(g, p.planes, p.plane, p.planes, p.plane);
            g.bias = bias ? (const uint8_t *)bias + (size_t)v0 * es : nullptr;
            g.bias_bf16 = prec == P_BF16; g.labels = labels; g.v0 = v0; g.V = out;
            g.lse = lse; g.drow = drow; g.planes = p.dz_planes; g.dz_plane = p.chunk;
            g.db_part = db ? (float *)(base + p.db) : nullptr;
            // chains as the forward pass cuts them, whatever is asked for: exp(z - lse) has to see one z
            const int r = ce_launch<kDz, false, false>(ox, ow, oz, g, true, s);
            if (r < 0) return r;
            n += r;
        }
        if (db && !db_last) {
            CeDb d = db_all;
            d.db = db + v0;
            d.cols = cols;
            launch_k(ce_db_kernel, ceil_div(cols, 32), 256, 0, s, d, (const CeHeader *)head);
            ++n;
        }
        if (dx) {
            CeGemm g{};
            CeOperand o{};  // written by TMA
            g.M = B; g.N = in; g.K = cols; g.head = head; g.b_k0 = v0;
            ce_segments(g, p.planes, p.chunk, p.planes, p.plane);
            g.splits = p.splits;  // a short last chunk may take fewer: it adds to the first partials only
            g.ld = p.dx_ld; g.out_split = (size_t)B * p.dx_ld;
            if (dx_direct && v0 + cols >= out) {
                g.out = dx; g.out_kind = kFinal; g.labels = labels; g.V = out;
                g.part_in = v0 > 0 ? (const float *)(base + p.dx) : nullptr;
                g.out_bf16 = prec == P_BF16;
                g.out_tma = g.out_bf16 && in % 8 == 0 && (reinterpret_cast<uintptr_t>(dx) & 15) == 0;
                if (g.out_tma) o = CeOperand{dx, B, in};
            } else {
                g.out = base + p.dx; g.out_kind = v0 > 0 ? kAdd : kStore;
            }
            const int r = ce_launch<kPartial, false, true>(oz, ow, o, g, prec == P_F32, s);
            if (r < 0) return r;
            n += r;
        }
        if (dW) {
            const int r = weight_gradient(v0, cols);
            if (r < 0) return r;
            n += r;
        }
    }
    if (!dx || dx_direct) {
        launch_k(ce_end_kernel, 148, 256, 0, s, (const CeHeader *)head, results);
        return n + 1;
    }
    return n + join_dx(prec, p, base, labels, results, B, in, out, db_all, db_last ? ceil_div(out, 32) : 0, s);
}

}  // namespace ddg

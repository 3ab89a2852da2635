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
// All four products run on one tcgen05 kernel.  What bounds it: 2NVD (forward) and 6NVD (backward) multiply-adds on the
// tensor cores; for a few rows the bytes of W.  Two CTAs of a cluster work on one 256 x 256 tile (cta_group::2): each
// loads half of A and half of B (32 KB for 64 values of K instead of 48 KB for two tiles of their own), so that the L2
// can feed the tensor cores; six such stages are in flight by TMA, and two accumulators (512 TMEM columns) let the
// epilogue of a tile run under the next tile's products.
//
// fp32 tensors are split into three bf16 terms each (x = h + m + l to 24 bits) and the products h h, h m, m h, m m, h l,
// l h are accumulated, smallest first: what is left out is below 2^-24 of the value.
#include <algorithm>

#include "common.cuh"
#include "conv_tc.h"
#include "lm_ops.h"
#include "tc_common.cuh"

namespace ddg {

namespace {

constexpr int kTile = 256;        // rows and columns of a tile of the CTA pair
constexpr int kHalf = 128;        // rows of A and of B that one CTA of the pair loads
constexpr int kKBox = 64;         // K values of a stage: 128 bytes of bf16, one swizzle row
constexpr int kStages = 6;
constexpr int kStageBytes = 2 * kHalf * kKBox * 2;  // per CTA: A half + B half
constexpr int kEpiWarps = 8;      // two per TMEM lane quarter, each half of the columns
constexpr int kThreads = 64 + 32 * kEpiWarps;
constexpr int kCeSmem = kStages * kStageBytes + 1024;
constexpr int kMaxSeg = 6;
constexpr float kLog2e = 1.4426950408889634f;

enum Mode { kLse, kDz, kPartial, kWeightGrad };

// What the workspace starts with.
struct CeHeader {
    int err;            // a bounded wait ran out: the kernels that write the results turn them into NaN
    unsigned ticket;    // blocks of the joining kernel that are done
    float scale;        // factor on dx and dW: upstream gradient / counted rows
    int pad[61];
};
static_assert(sizeof(CeHeader) == 256, "the buffers behind the header stay aligned");

struct CeGemm {
    int M, N;                 // rows of A, rows of B (columns of the result)
    int kblocks, n_seg;       // 64-wide K blocks per segment; segments: pairs of bf16 terms
    int a_off[kMaxSeg], b_off[kMaxSeg];  // where a segment's term starts: in K (K-major operand) or in M / N
    int a_r0, b_r0, b_k0;     // coordinates of the first row of A and of B and of B's first K value
    int tiles_m, tiles_n, splits, group_m;
    CeHeader *head;
    // kLse, kDz
    const void *bias;         // nullable, at column 0 of this launch
    int bias_bf16;
    const int *labels;        // label of every row; columns are v0 + n
    int v0, V;
    float2 *part;             // kLse: [2 tiles_n][M] (maximum, sum)
    float *zlab;              // kLse: logit of the label
    const float *lse, *drow;  // kDz
    bf16 *dz;                 // kDz: [M][planes * dz_plane]
    int planes, dz_plane;
    float *db_part;           // kDz, nullable: [ceil(M / 32)][dz_plane]
    // kPartial: fp32 [splits][M][ld];  kWeightGrad: [M][ld] in the element type
    void *out;
    size_t out_split;
    int ld, accumulate, out_bf16, out_vec;
};

__device__ __forceinline__ uint32_t cluster_rank() { uint32_t r; asm("mov.u32 %0, %%cluster_ctarank;" : "=r"(r)); return r; }
__device__ __forceinline__ void cluster_sync() {
    asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
__device__ __forceinline__ uint32_t map_rank(uint32_t addr, uint32_t rank) {
    uint32_t r;
    asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(addr), "r"(rank));
    return r;
}
__device__ __forceinline__ void mbar_arrive_remote(uint32_t cluster_addr) {
    asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0];" ::"r"(cluster_addr) : "memory");
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
// arrives on the barrier at this offset in both CTAs when the MMAs issued so far are done
__device__ __forceinline__ void commit_pair(uint32_t bar) {
    asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;"
                 ::"r"(bar), "h"((uint16_t)3) : "memory");
}
__device__ __forceinline__ float exp2_approx(float v) { float r; asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(v)); return r; }

// Which tile a work item is: all tiles of a split, in bands of group_m tile rows that are walked column by column, so
// that the operands of the tiles in flight stay in the L2.
struct CeItem { int split, m, n, kb0, kb1; };
__device__ __forceinline__ CeItem ce_item(const CeGemm &g, int item) {
    CeItem it;
    const int per = g.tiles_m * g.tiles_n;
    it.split = item / per;
    int r = item - it.split * per;
    const int band = r / (g.group_m * g.tiles_n);
    r -= band * g.group_m * g.tiles_n;
    const int rows = min(g.group_m, g.tiles_m - band * g.group_m);
    it.n = r / rows;
    it.m = band * g.group_m + r - it.n * rows;
    const int kb = g.kblocks * g.n_seg;
    it.kb0 = (int)((long long)kb * it.split / g.splits);
    it.kb1 = (int)((long long)kb * (it.split + 1) / g.splits);
    return it;
}

// 32 columns of one row, v[0..32) in two halves, to the three places a value can go
__device__ __forceinline__ uint32_t pack2(float a, float b) {
    const __nv_bfloat162 h = __floats2bfloat162_rn(a, b);
    return *reinterpret_cast<const uint32_t *>(&h);
}
__device__ __forceinline__ float bf16_round(float v) { return __bfloat162float(__float2bfloat16_rn(v)); }

__device__ __forceinline__ void load_bias32(const CeGemm &g, int c0, float (&b)[32]) {
    // every lane reads the same 32 values (one transaction each); columns past the vocabulary are masked by the caller
#pragma unroll
    for (int j = 0; j < 32; ++j) {
        const int c = min(c0 + j, g.N - 1);
        b[j] = g.bias_bf16 ? __bfloat162float(((const bf16 *)g.bias)[c]) : ((const float *)g.bias)[c];
    }
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

template <int MODE>
__device__ __forceinline__ void ce_epilogue(const CeGemm &g, const CeItem &it, uint32_t acc, int quarter, int half, int rank, int lane,
                                            uint32_t release_bar) {
    const int row = it.m * kTile + rank * kHalf + 32 * quarter + lane;
    const int col0 = it.n * kTile + half * kHalf;
    const uint32_t taddr = acc + ((uint32_t)(32 * quarter) << 16) + (uint32_t)(half * kHalf);
    const bool live = row < g.M;
    float top = -INFINITY, sum = 0.f, lse = 0.f, weight = 0.f;
    int label = -1;
    if ((MODE == kLse || MODE == kDz) && live) {
        const int y = g.labels[row];
        label = y >= 0 && y < g.V ? y - g.v0 : -1 - kTile;  // column of this launch (a label of another chunk meets none)
        if (MODE == kDz) {
            lse = g.lse[row];
            weight = y >= 0 && y < g.V ? (g.drow ? g.drow[row] : 1.f) : 0.f;
        }
    }
#pragma unroll 1
    for (int c = 0; c < kHalf; c += 32) {
        float v[32];
        tc_ld32(taddr + (uint32_t)c, reinterpret_cast<float(&)[16]>(v[0]), reinterpret_cast<float(&)[16]>(v[16]));
        tc_wait_ld();
        if (c + 32 == kHalf) {  // the accumulator is read: the next tile's products may overwrite it
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive_remote(release_bar);
        }
        const int col = col0 + c;
        if (MODE == kLse || MODE == kDz) {
            if (g.bias) {
                float b[32];
                load_bias32(g, col, b);
#pragma unroll
                for (int j = 0; j < 32; ++j) v[j] += b[j];
            }
        }
        if (MODE == kLse) {
            if (col + 32 > g.N) {
#pragma unroll
                for (int j = 0; j < 32; ++j)
                    if (col + j >= g.N) v[j] = -INFINITY;
            }
            float m = v[0];
#pragma unroll
            for (int j = 1; j < 32; ++j) m = fmaxf(m, v[j]);
            m = fmaxf(top, m);
            const float ref = m == -INFINITY ? 0.f : m;  // nothing but -inf so far
            float s0 = sum * exp2_approx((top - ref) * kLog2e), s1 = 0.f;
#pragma unroll
            for (int j = 0; j < 32; j += 2) {
                s0 += exp2_approx((v[j] - ref) * kLog2e);
                s1 += exp2_approx((v[j + 1] - ref) * kLog2e);
            }
            top = m;
            sum = s0 + s1;
            if (label >= col && label < col + 32) {
                float z = 0.f;
#pragma unroll
                for (int j = 0; j < 32; ++j)
                    if (label == col + j) z = v[j];
                g.zlab[row] = z;
            }
        } else if (MODE == kDz) {
#pragma unroll
            for (int j = 0; j < 32; ++j) {
                const float p = exp2_approx((v[j] - lse) * kLog2e) - (label == col + j ? 1.f : 0.f);
                // a row that does not count gives exact zeros whatever its logits are; so do columns past the vocabulary
                v[j] = weight != 0.f && col + j < g.N ? p * weight : 0.f;
            }
            if (g.db_part) {  // rows that are not there hold zeros
                float t[32];
#pragma unroll
                for (int j = 0; j < 32; ++j) t[j] = v[j];
                const float cs = column_sums(t, lane);
                const int block = (it.m * kTile + rank * kHalf) / 32 + quarter;
                if (block * 32 < g.M) g.db_part[(size_t)block * g.dz_plane + col + lane] = cs;
            }
            if (live) {
                bf16 *dst = g.dz + (size_t)row * g.planes * g.dz_plane + col;
                for (int p = 0; p < g.planes; ++p, dst += g.dz_plane) {
                    uint32_t w[16];
#pragma unroll
                    for (int j = 0; j < 16; ++j) w[j] = pack2(v[2 * j], v[2 * j + 1]);
                    st_global_32(dst, reinterpret_cast<const uint32_t(&)[8]>(w[0]));
                    st_global_32(dst + 16, reinterpret_cast<const uint32_t(&)[8]>(w[8]));
#pragma unroll
                    for (int j = 0; j < 32; ++j) v[j] -= bf16_round(v[j]);
                }
            }
        } else if (MODE == kPartial) {
            if (live) {
                float *dst = (float *)g.out + it.split * g.out_split + (size_t)row * g.ld + col;
#pragma unroll
                for (int j = 0; j < 32; j += 4) {
                    if (col + j < g.ld) {  // ld is a multiple of 4
                        float4 q = make_float4(v[j], v[j + 1], v[j + 2], v[j + 3]);
                        if (g.accumulate) {
                            const float4 o = *reinterpret_cast<const float4 *>(dst + j);
                            q = make_float4(q.x + o.x, q.y + o.y, q.z + o.z, q.w + o.w);
                        }
                        *reinterpret_cast<float4 *>(dst + j) = q;
                    }
                }
            }
        } else {
            if (live) {
                const float scale = g.head->scale;
#pragma unroll
                for (int j = 0; j < 32; ++j) v[j] *= scale;
                const size_t at = (size_t)row * g.ld + col;
                if (g.out_bf16) {
                    bf16 *dst = (bf16 *)g.out + at;
                    if (g.out_vec) {  // ld is a multiple of 8
#pragma unroll
                        for (int j = 0; j < 32; j += 8)
                            if (col + j < g.ld)
                                *reinterpret_cast<uint4 *>(dst + j) = make_uint4(pack2(v[j], v[j + 1]), pack2(v[j + 2], v[j + 3]),
                                                                                 pack2(v[j + 4], v[j + 5]), pack2(v[j + 6], v[j + 7]));
                    } else {
#pragma unroll
                        for (int j = 0; j < 32; ++j)
                            if (col + j < g.ld) dst[j] = __float2bfloat16_rn(v[j]);
                    }
                } else {
                    float *dst = (float *)g.out + at;
                    if (g.out_vec) {  // ld is a multiple of 4
#pragma unroll
                        for (int j = 0; j < 32; j += 4)
                            if (col + j < g.ld) *reinterpret_cast<float4 *>(dst + j) = make_float4(v[j], v[j + 1], v[j + 2], v[j + 3]);
                    } else {
#pragma unroll
                        for (int j = 0; j < 32; ++j)
                            if (col + j < g.ld) dst[j] = v[j];
                    }
                }
            }
        }
    }
    if (MODE == kLse && live) g.part[(size_t)(2 * it.n + half) * g.M + row] = make_float2(top, sum);
}

// A_MN / B_MN: the operand lies with M / N innermost (its rows are K values) instead of K.
template <int MODE, bool A_MN, bool B_MN>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kThreads, 1)
ce_gemm_kernel(const __grid_constant__ CUtensorMap map_a, const __grid_constant__ CUtensorMap map_b, const __grid_constant__ CeGemm g) {
    extern __shared__ uint8_t smem_raw[];
    __shared__ uint64_t full[kStages], empty[kStages], acc_full[2], acc_empty[2];
    __shared__ uint32_t tmem_holder;
    __shared__ int abort_flag;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t rank = cluster_rank();
    const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u;
    const Waiter wt{&abort_flag, &g.head->err, kSpinLimit};
    if (threadIdx.x == 0) {
        for (int i = 0; i < kStages; ++i) { mbar_init(smem_u32(&full[i]), 1); mbar_init(smem_u32(&empty[i]), 1); }
        for (int i = 0; i < 2; ++i) { mbar_init(smem_u32(&acc_full[i]), 1); mbar_init(smem_u32(&acc_empty[i]), 2 * kEpiWarps); }
        abort_flag = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 1) {
        asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&tmem_holder)), "r"(512u) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
    }
    pdl_launch();
    pdl_wait();
    tc_fence_before();
    __syncthreads();
    cluster_sync();  // both CTAs' barriers are ready
    tc_fence_after();
    const uint32_t tmem = tmem_holder;
    const int n_items = g.tiles_m * g.tiles_n * g.splits;
    const int first = blockIdx.x >> 1, step = gridDim.x >> 1;

    if (warp == 0) {
        if (lane == 0) {  // loads
            bool ok = true;
            uint32_t n = 0;
            for (int item = first; item < n_items && ok; item += step) {
                const CeItem it = ce_item(g, item);
                const int m0 = it.m * kTile + (int)rank * kHalf, n0 = it.n * kTile + (int)rank * kHalf;
                int seg = it.kb0 / g.kblocks, kb = it.kb0 - seg * g.kblocks;
                for (int i = it.kb0; i < it.kb1; ++i, ++n) {
                    const uint32_t s = n % kStages, ph = (n / kStages) & 1u;
                    if (!mbar_wait(smem_u32(&empty[s]), ph ^ 1u, wt, 51)) { ok = false; break; }
                    if (rank == 0) mbar_expect_tx(smem_u32(&full[s]), 2u * kStageBytes);
                    const uint32_t bar = map_rank(smem_u32(&full[s]), 0);
                    const uint32_t a = base + s * kStageBytes, b = a + kStageBytes / 2;
                    const int k = kb * kKBox;
                    if (A_MN) {
                        tma_load_pair(a, &map_a, bar, g.a_off[seg] + m0, k);
                        tma_load_pair(a + 8192, &map_a, bar, g.a_off[seg] + m0 + 64, k);
                    } else {
                        tma_load_pair(a, &map_a, bar, g.a_off[seg] + k, g.a_r0 + m0);
                    }
                    if (B_MN) {
                        tma_load_pair(b, &map_b, bar, g.b_off[seg] + n0, g.b_k0 + k);
                        tma_load_pair(b + 8192, &map_b, bar, g.b_off[seg] + n0 + 64, g.b_k0 + k);
                    } else {
                        tma_load_pair(b, &map_b, bar, g.b_off[seg] + k, g.b_r0 + n0);
                    }
                    if (++kb == g.kblocks) { kb = 0; ++seg; }
                }
            }
            if (!ok)
                for (int i = 0; i < 2000; ++i) __nanosleep(100);  // copies in flight land before the CTA can exit
        }
        __syncwarp();
    } else if (warp == 1) {
        if (rank == 0 && lane == 0) {  // products, for both CTAs
            const uint32_t idesc = (1u << 4) | (1u << 7) | (1u << 10) | (A_MN ? 1u << 15 : 0u) | (B_MN ? 1u << 16 : 0u) |
                                   ((uint32_t)(kTile >> 3) << 17) | ((uint32_t)(kTile >> 4) << 24);
            bool ok = true;
            uint32_t n = 0, t = 0;
            for (int item = first; item < n_items && ok; item += step, ++t) {
                const CeItem it = ce_item(g, item);
                const uint32_t acc = t & 1u;
                if (!mbar_wait(smem_u32(&acc_empty[acc]), ((t >> 1) & 1u) ^ 1u, wt, 52)) break;
                tc_fence_after();
                for (int i = it.kb0; i < it.kb1; ++i, ++n) {
                    const uint32_t s = n % kStages, ph = (n / kStages) & 1u;
                    if (!mbar_wait(smem_u32(&full[s]), ph, wt, 53)) { ok = false; break; }
                    tc_fence_after();
                    const uint32_t a = base + s * kStageBytes, b = a + kStageBytes / 2;
                    // K-major: 16 K values are 32 bytes of a swizzle row.  MN-major: 16 rows of 128 bytes; the next 64
                    // of the 128 M / N values lie 8 KB further.
                    const uint64_t ad = A_MN ? make_desc(a, 1024, 2u, 8192) : make_desc(a, 1024, 2u);
                    const uint64_t bd = B_MN ? make_desc(b, 1024, 2u, 8192) : make_desc(b, 1024, 2u);
#pragma unroll
                    for (int k = 0; k < kKBox / 16; ++k)
                        mma_pair(tmem + acc * kTile, ad + (A_MN ? 128 : 2) * k, bd + (B_MN ? 128 : 2) * k, idesc, i > it.kb0 || k > 0);
                    commit_pair(smem_u32(&empty[s]));
                }
                if (ok) commit_pair(smem_u32(&acc_full[acc]));
            }
        }
        __syncwarp();
    } else {
        const int quarter = warp & 3, half = (warp - 2) >> 2;
        uint32_t t = 0;
        for (int item = first; item < n_items; item += step, ++t) {
            const CeItem it = ce_item(g, item);
            const uint32_t acc = t & 1u;
            bool ok = mbar_wait(smem_u32(&acc_full[acc]), (t >> 1) & 1u, wt, 54);
            if (!__all_sync(0xffffffffu, ok)) break;
            tc_fence_after();
            ce_epilogue<MODE>(g, it, tmem + acc * kTile, quarter, half, (int)rank, lane, map_rank(smem_u32(&acc_empty[acc]), 0));
        }
    }
    tc_fence_before();
    __syncthreads();
    cluster_sync();  // no MMA of the pair reads this CTA's shared memory or writes its TMEM any more
    if (warp == 1) {
        tc_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512u) : "memory");
    }
    cluster_sync();
}

// ---- joining the forward pass ----------------------------------------------------------------------------------------
// rows rows per block of 256 threads, the other 256 / rows threads share a row's pieces.  The mean is taken by the block
// that finishes last, over the blocks' sums in index order.
__global__ void __launch_bounds__(256) ce_join_kernel(const float2 *__restrict__ part, int n_part, const float *__restrict__ zlab, const int *__restrict__ labels,
                                                      float *__restrict__ loss, float *__restrict__ row_loss, float *__restrict__ lse_out,
                                                      double *__restrict__ sums, CeHeader *head, int B, int V, int rows) {
    __shared__ float sm[256], ss[256];
    __shared__ double bl[32];
    __shared__ int bc[32], last;
    pdl_launch();
    pdl_wait();
    const int r = threadIdx.x & (rows - 1), t0 = threadIdx.x / rows, lanes = 256 / rows;
    const int row = blockIdx.x * rows + r;
    float m = -INFINITY, s = 0.f;
    if (row < B) {
        for (int t = t0; t < n_part; t += 4 * lanes) {  // four loads in flight
            float2 q[4];
#pragma unroll
            for (int u = 0; u < 4; ++u) q[u] = t + u * lanes < n_part ? part[(size_t)(t + u * lanes) * B + row] : make_float2(-INFINITY, 0.f);
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                const float top = fmaxf(m, q[u].x), ref = top == -INFINITY ? 0.f : top;
                s = s * expf(m - ref) + q[u].y * expf(q[u].x - ref);
                m = top;
            }
        }
    }
    sm[threadIdx.x] = m;
    ss[threadIdx.x] = s;
    __syncthreads();
    for (int o = lanes / 2; o > 0; o >>= 1) {
        if (t0 < o) {
            const int i = threadIdx.x, j = i + o * rows;
            const float top = fmaxf(sm[i], sm[j]), ref = top == -INFINITY ? 0.f : top;
            ss[i] = ss[i] * expf(sm[i] - ref) + ss[j] * expf(sm[j] - ref);
            sm[i] = top;
        }
        __syncthreads();
    }
    const bool failed = head->err != 0;
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
        __shared__ double fa[256], fc[256];
        __threadfence();
        double a = 0.0, c = 0.0;
        for (int i = threadIdx.x; i < (int)gridDim.x; i += 256) { a += __ldcg(sums + 2 * i); c += __ldcg(sums + 2 * i + 1); }
        fa[threadIdx.x] = a;
        fc[threadIdx.x] = c;
        __syncthreads();
        for (int o = 128; o > 0; o >>= 1) {
            if ((int)threadIdx.x < o) { fa[threadIdx.x] += fa[threadIdx.x + o]; fc[threadIdx.x] += fc[threadIdx.x + o]; }
            __syncthreads();
        }
        if (threadIdx.x == 0) *loss = (float)(fa[0] / fmax(fc[0], 1.0));
    }
}

// ---- operands that TMA cannot read in place --------------------------------------------------------------------------
// dst [rows][planes * plane] bf16: term p of column c at p * plane + c, zero past `cols`.  labels (nullable): rows that do
// not count become zero, so that what stands in them (NaN among it) stays out of dW.  When `count` is set the
// last block sets the scale of the backward pass instead of copying.
template <typename T>
__global__ void __launch_bounds__(256) ce_pack_kernel(const T *__restrict__ src, bf16 *__restrict__ dst, const int *__restrict__ labels, int rows, int cols,
                                                      int plane, int planes, int V, CeHeader *head, int count, int mean, const float *__restrict__ dloss) {
    pdl_launch();
    pdl_wait();
    if (count && blockIdx.x == gridDim.x - 1) {
        __shared__ int part[256];
        int n = 0;
        if (mean)
            for (int i = threadIdx.x; i < rows; i += 256) n += labels[i] >= 0 && labels[i] < V;
        part[threadIdx.x] = n;
        __syncthreads();
        for (int o = 128; o > 0; o >>= 1) {
            if ((int)threadIdx.x < o) part[threadIdx.x] += part[threadIdx.x + o];
            __syncthreads();
        }
        if (threadIdx.x == 0) head->scale = mean ? (dloss ? *dloss : 1.f) / (float)max(part[0], 1) : 1.f;
        return;
    }
    // eight columns per step; plane is a multiple of 8
    const size_t total = (size_t)rows * (plane / 8);
    const size_t blocks = gridDim.x - (count ? 1 : 0);
    const bool vec = cols % (16 / (int)sizeof(T)) == 0 && (reinterpret_cast<uintptr_t>(src) & 15) == 0 && cols == plane;
    for (size_t i = (size_t)blockIdx.x * 256 + threadIdx.x; i < total; i += blocks * 256) {
        const size_t row = i / (plane / 8);
        const int c = (int)(i - row * (plane / 8)) * 8;
        float v[8];
        bool live = true;
        if (labels) { const int y = labels[row]; live = y >= 0 && y < V; }
        if (live && vec) {
            if (sizeof(T) == 2) {
                load_f<T, 8>(src + row * cols + c, v);
            } else {
                load_f<T, 4>(src + row * cols + c, reinterpret_cast<float(&)[4]>(v[0]));
                load_f<T, 4>(src + row * cols + c + 4, reinterpret_cast<float(&)[4]>(v[4]));
            }
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] = live && c + j < cols ? to_f(src[row * cols + c + j]) : 0.f;
        }
        for (int p = 0; p < planes; ++p) {
            *reinterpret_cast<uint4 *>(dst + row * planes * plane + (size_t)p * plane + c) =
                make_uint4(pack2(v[0], v[1]), pack2(v[2], v[3]), pack2(v[4], v[5]), pack2(v[6], v[7]));
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                // an infinity or NaN stays in the first term alone (inf - inf would spread NaN into its row's others)
                const float h = bf16_round(v[j]);
                v[j] = isinf(h) || isnan(h) ? 0.f : v[j] - h;
            }
        }
    }
}

// ---- ends of the backward pass ---------------------------------------------------------------------------------------
// db[v0 + c] = scale * sum over row blocks of db_part[block][c], blocks in index order per thread, threads in index order
__global__ void __launch_bounds__(256) ce_db_kernel(const float *__restrict__ db_part, int blocks, int plane, float *__restrict__ db, int cols, const CeHeader *head) {
    __shared__ double fold[8][32];
    pdl_launch();
    pdl_wait();
    const int lane = threadIdx.x & 31, w = threadIdx.x >> 5, c = blockIdx.x * 32 + lane;
    double a = 0.0;
    if (c < cols)
        for (int b = w; b < blocks; b += 8) a += (double)db_part[(size_t)b * plane + c];
    fold[w][lane] = a;
    __syncthreads();
    if (w == 0 && c < cols) {
        for (int i = 1; i < 8; ++i) a += fold[i][lane];
        db[c] = head->err ? __int_as_float(0x7fffffff) : (float)(a * (double)head->scale);
    }
}

// dx[n][c] = scale * sum_s part[s][n][c]; rows that do not count are zero
template <typename T>
__global__ void __launch_bounds__(256) ce_dx_kernel(const float *__restrict__ part, int splits, size_t split_stride, int ld, const int *__restrict__ labels, T *__restrict__ dx,
                                                    int B, int in, int V, int vec, const CeHeader *head, void *dW, int dw_bf16) {
    pdl_launch();
    pdl_wait();
    const bool failed = head->err != 0;
    const float scale = head->scale, nan = __int_as_float(0x7fffffff);
    if (failed && dW && blockIdx.x == 0 && threadIdx.x == 0) {
        if (dw_bf16) *(bf16 *)dW = __float2bfloat16_rn(nan); else *(float *)dW = nan;
    }
    if (!dx) return;
    const size_t total = (size_t)B * (ld / 4);
    for (size_t i = (size_t)blockIdx.x * 256 + threadIdx.x; i < total; i += (size_t)gridDim.x * 256) {
        const size_t row = i / (ld / 4);
        const int c = (int)(i - row * (ld / 4)) * 4;
        const int y = labels[row];
        float4 a = make_float4(0.f, 0.f, 0.f, 0.f);
        if (y >= 0 && y < V) {
            for (int s = 0; s < splits; ++s) {
                const float4 q = *reinterpret_cast<const float4 *>(part + s * split_stride + row * ld + c);
                a.x += q.x; a.y += q.y; a.z += q.z; a.w += q.w;
            }
        }
        float v[4] = {a.x * scale, a.y * scale, a.z * scale, a.w * scale};
        if (failed) v[0] = v[1] = v[2] = v[3] = nan;
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

int sm_count() {
    int dev = 0, n = 148;
    if (cudaGetDevice(&dev) == cudaSuccess) cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev);
    return n;
}

// A chunk of the vocabulary: dz of all rows for at most kDzBytes, at least one tile wide.  The chunk is written once and
// read twice; larger chunks mean fewer passes over the fp32 partial sums of dx.
constexpr size_t kDzBytes = (size_t)256 << 20;
constexpr int kPairs = 74;  // CTA pairs of the GPU: the splits of a plan (and with them the workspace) go by this number

struct CePlan {
    int planes, plane;       // terms of an element, columns of a term in a packed operand
    int dz_planes, chunk;    // terms of dz, columns of a chunk
    int tiles_m, n_part;
    int splits, dx_ld;
    bool pack_x, pack_w;
    size_t part, zlab, sums, x, w, dz, db, dx, bytes;
};

CePlan ce_plan(int prec, int B, int in, int out, bool backward, bool dw_f32) {
    CePlan p{};
    p.planes = prec == P_F32 ? 3 : 1;
    p.plane = prec == P_F32 ? up(in, 64) : up(in, 8);
    p.pack_w = prec == P_F32 || in % 8 != 0;
    p.pack_x = p.pack_w || backward;
    // an fp32 dW of bf16 operands gets 16 bits of dz (two terms), as the fully connected layer's loss gradient does; a bf16
    // dW or dx is rounded to 8 bits itself and takes dz rounded once to bf16
    p.dz_planes = prec == P_F32 ? 3 : (dw_f32 ? 2 : 1);
    p.tiles_m = (B + kTile - 1) / kTile;
    p.n_part = 2 * ((out + kTile - 1) / kTile);
    size_t at = sizeof(CeHeader);
    auto take = [&](size_t bytes) { const size_t r = at; at += up256(bytes); return r; };
    if (!backward) {
        p.part = take((size_t)p.n_part * B * sizeof(float2));
        p.zlab = take((size_t)B * 4);
        p.sums = take((size_t)B * 16);
    }
    if (p.pack_x) p.x = take((size_t)B * p.planes * p.plane * 2);
    if (p.pack_w) p.w = take((size_t)out * p.planes * p.plane * 2);
    if (backward) {
        const size_t fit = kDzBytes / ((size_t)B * p.dz_planes * 2) / kTile * kTile;
        p.chunk = (int)std::min<size_t>((size_t)up(out, kTile), std::max<size_t>(kTile, fit));
        p.dx_ld = up(in, 4);
        const int tiles = p.tiles_m * ((in + kTile - 1) / kTile);
        const int kb = std::min(p.chunk, up(out, kKBox)) / kKBox * (prec == P_F32 ? 6 : 1);
        p.splits = std::max(1, std::min(kPairs / tiles, kb / 8));
        p.dz = take((size_t)B * p.dz_planes * p.chunk * 2);
        p.db = take((size_t)((B + 31) / 32) * p.chunk * 4);
        p.dx = take((size_t)p.splits * B * p.dx_ld * 4);
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

template <int MODE, bool A_MN, bool B_MN>
int ce_launch(const CUtensorMap &a, const CUtensorMap &b, CeGemm &g, const Launch &s) {
    g.tiles_m = (g.M + kTile - 1) / kTile;
    g.tiles_n = (g.N + kTile - 1) / kTile;
    if (g.splits < 1) g.splits = 1;
    g.group_m = 16;
    const long items = (long)g.tiles_m * g.tiles_n * g.splits;
    if (items > 0x7fffffff) return -1;
    static thread_local int ready_dev = -1;  // the attribute belongs to a device
    int dev = 0;
    cudaGetDevice(&dev);
    if (ready_dev != dev) {
        if (cudaFuncSetAttribute(ce_gemm_kernel<MODE, A_MN, B_MN>, cudaFuncAttributeMaxDynamicSharedMemorySize, kCeSmem) != cudaSuccess) return -1;
        ready_dev = dev;
    }
    const int pairs = (int)std::min<long>(items, sm_count() / 2);
    Launch plain(s.s, 0, s.shared, s.err);
    launch_k(ce_gemm_kernel<MODE, A_MN, B_MN>, 2 * pairs, kThreads, kCeSmem, plain, a, b, g);
    return 1;
}

// terms of A and of B that are multiplied, smallest products first
void ce_segments(CeGemm &g, int a_planes, int a_plane, int b_planes, int b_plane) {
    g.n_seg = 0;
    auto add = [&](int i, int j) {
        if (i < a_planes && j < b_planes) { g.a_off[g.n_seg] = i * a_plane; g.b_off[g.n_seg] = j * b_plane; ++g.n_seg; }
    };
    add(2, 0); add(0, 2); add(1, 1); add(1, 0); add(0, 1); add(0, 0);
}

int grid_for(size_t threads) { return (int)std::max<size_t>(1, std::min<size_t>((threads + 255) / 256, 148 * 8)); }

int pack(int prec, const void *src, void *dst, const int *labels, int rows, int cols, const CePlan &p, int V, CeHeader *head, int count, int mean,
         const float *dloss, const Launch &s) {
    const int grid = grid_for((size_t)rows * (p.plane / 8)) + (count ? 1 : 0);
    if (prec == P_BF16)
        launch_k(ce_pack_kernel<bf16>, grid, 256, 0, s, (const bf16 *)src, (bf16 *)dst, labels, rows, cols, p.plane, p.planes, V, head, count, mean, dloss);
    else
        launch_k(ce_pack_kernel<float>, grid, 256, 0, s, (const float *)src, (bf16 *)dst, labels, rows, cols, p.plane, p.planes, V, head, count, mean, dloss);
    return 1;
}

}  // namespace

bool linear_ce_in_place(int prec, int in) { return prec == P_BF16 && in % 8 == 0; }

size_t linear_ce_workspace_bytes(int prec, int B, int in, int out, int backward) {
    return std::max(ce_plan(prec, B, in, out, backward != 0, false).bytes, ce_plan(prec, B, in, out, backward != 0, true).bytes);
}

int launch_linear_ce_fwd(int prec, const void *x, const void *W, const void *bias, const int *labels, float *loss, float *row_loss, float *lse,
                         void *ws, int B, int in, int out, Launch s) {
    const CePlan p = ce_plan(prec, B, in, out, false, false);
    uint8_t *base = (uint8_t *)ws;
    CeHeader *head = (CeHeader *)base;
    const Launch plain(s.s, 0, s.shared, s.err);
    if (cudaMemsetAsync(head, 0, sizeof(CeHeader), s) != cudaSuccess) return -1;
    int n = 0;
    if (p.pack_x) { n += pack(prec, x, base + p.x, nullptr, B, in, p, out, head, 0, 0, nullptr, plain); x = base + p.x; }
    if (p.pack_w) { n += pack(prec, W, base + p.w, nullptr, out, in, p, out, head, 0, 0, nullptr, plain); W = base + p.w; }
    const int cols = p.pack_w ? p.planes * p.plane : in;
    CUtensorMap ma, mb;
    if (!ce_map(x, B, cols, cols, kHalf, &ma) || !ce_map(W, out, cols, cols, kHalf, &mb)) return -1;
    CeGemm g{};
    g.M = B; g.N = out; g.kblocks = (p.plane + kKBox - 1) / kKBox; g.head = head;
    ce_segments(g, p.planes, p.plane, p.planes, p.plane);
    g.bias = bias; g.bias_bf16 = prec == P_BF16; g.labels = labels; g.V = out;
    g.part = (float2 *)(base + p.part); g.zlab = (float *)(base + p.zlab);
    const int r = ce_launch<kLse, false, false>(ma, mb, g, s);
    if (r < 0) return r;
    int rows = 1;
    while (rows < 32 && rows < B) rows *= 2;
    launch_k(ce_join_kernel, (B + rows - 1) / rows, 256, 0, plain, (const float2 *)g.part, p.n_part, (const float *)g.zlab, labels, loss, row_loss, lse,
             (double *)(base + p.sums), head, B, out, rows);
    return n + r + 1;
}

int launch_linear_ce_bwd(int prec, const void *x, const void *W, const void *bias, const int *labels, const float *lse, const float *dloss,
                         const float *drow, void *dx, void *dW, float *db, void *ws, int B, int in, int out, int dw_f32, Launch s) {
    const CePlan p = ce_plan(prec, B, in, out, true, dw_f32 != 0);
    uint8_t *base = (uint8_t *)ws;
    CeHeader *head = (CeHeader *)base;
    const Launch plain(s.s, 0, s.shared, s.err);
    if (cudaMemsetAsync(head, 0, sizeof(CeHeader), s) != cudaSuccess) return -1;
    int n = pack(prec, x, base + p.x, labels, B, in, p, out, head, 1, drow == nullptr, dloss, plain);
    const void *xp = base + p.x;
    if (p.pack_w) { n += pack(prec, W, base + p.w, nullptr, out, in, p, out, head, 0, 0, nullptr, plain); W = base + p.w; }
    const int x_cols = p.planes * p.plane, w_cols = p.pack_w ? p.planes * p.plane : in;
    const int dz_cols = p.dz_planes * p.chunk;
    bf16 *dz = (bf16 *)(base + p.dz);
    CUtensorMap mx, mw, mx_mn, mw_mn, mz, mz_mn;
    if (!ce_map(xp, B, x_cols, x_cols, kHalf, &mx) || !ce_map(W, out, w_cols, w_cols, kHalf, &mw) || !ce_map(xp, B, x_cols, x_cols, kKBox, &mx_mn) ||
        !ce_map(W, out, w_cols, w_cols, kKBox, &mw_mn) || !ce_map(dz, B, dz_cols, dz_cols, kHalf, &mz) || !ce_map(dz, B, dz_cols, dz_cols, kKBox, &mz_mn))
        return -1;
    const int es = prec == P_BF16 ? 2 : 4;
    for (int v0 = 0; v0 < out; v0 += p.chunk) {
        const int cols = std::min(p.chunk, out - v0);
        {
            CeGemm g{};
            g.M = B; g.N = cols; g.kblocks = (p.plane + kKBox - 1) / kKBox; g.head = head; g.b_r0 = v0;
            ce_segments(g, p.planes, p.plane, p.planes, p.plane);
            g.bias = bias ? (const uint8_t *)bias + (size_t)v0 * es : nullptr;
            g.bias_bf16 = prec == P_BF16; g.labels = labels; g.v0 = v0; g.V = out;
            g.lse = lse; g.drow = drow; g.dz = dz; g.planes = p.dz_planes; g.dz_plane = p.chunk;
            g.db_part = db ? (float *)(base + p.db) : nullptr;
            const int r = ce_launch<kDz, false, false>(mx, mw, g, s);
            if (r < 0) return r;
            n += r;
        }
        if (db) {
            launch_k(ce_db_kernel, ceil_div(cols, 32), 256, 0, plain, (const float *)(base + p.db), (B + 31) / 32, p.chunk, db + v0, cols, (const CeHeader *)head);
            ++n;
        }
        if (dx) {
            CeGemm g{};
            g.M = B; g.N = in; g.kblocks = (cols + kKBox - 1) / kKBox; g.head = head; g.b_k0 = v0;
            ce_segments(g, p.planes, p.chunk, p.planes, p.plane);
            g.splits = std::min(p.splits, g.kblocks * g.n_seg);  // a short last chunk adds to the first partials only
            g.out = base + p.dx; g.ld = p.dx_ld; g.out_split = (size_t)B * p.dx_ld; g.accumulate = v0 > 0;
            const int r = ce_launch<kPartial, false, true>(mz, mw_mn, g, s);
            if (r < 0) return r;
            n += r;
        }
        if (dW) {
            const bool out_bf16 = prec == P_BF16 && !dw_f32;
            const int oe = out_bf16 ? 2 : 4;
            CeGemm g{};
            g.M = cols; g.N = in; g.kblocks = (B + kKBox - 1) / kKBox; g.head = head;
            ce_segments(g, p.dz_planes, p.chunk, p.planes, p.plane);
            g.out = (uint8_t *)dW + (size_t)v0 * in * oe; g.ld = in; g.out_bf16 = out_bf16;
            g.out_vec = (in * oe) % 16 == 0 && (reinterpret_cast<uintptr_t>(dW) & 15) == 0;
            const int r = ce_launch<kWeightGrad, true, true>(mz_mn, mx_mn, g, s);
            if (r < 0) return r;
            n += r;
        }
    }
    const int grid = dx ? grid_for((size_t)B * (p.dx_ld / 4)) : 1;
    const int vec = in % 4 == 0 && (reinterpret_cast<uintptr_t>(dx) & (4 * es - 1)) == 0;
    const int dw_bf16 = prec == P_BF16 && !dw_f32;
    if (prec == P_BF16)
        launch_k(ce_dx_kernel<bf16>, grid, 256, 0, plain, (const float *)(base + p.dx), p.splits, (size_t)B * p.dx_ld, p.dx_ld, labels, (bf16 *)dx, B, in, out, vec,
                 (const CeHeader *)head, dW, dw_bf16);
    else
        launch_k(ce_dx_kernel<float>, grid, 256, 0, plain, (const float *)(base + p.dx), p.splits, (size_t)B * p.dx_ld, p.dx_ld, labels, (float *)dx, B, in, out, vec,
                 (const CeHeader *)head, dW, dw_bf16);
    return n + 1;
}

}  // namespace ddg

// The vocabulary projection for a few rows (at most 64), part of linear_ce.cu.
//
// With n rows a value of W is multiplied n times: for n <= 64 the bytes of W bound the time.  So W is the operand with the
// 128 rows of an MMA (vocabulary entries, or in the product for dx the columns of W) and the rows of x are its 16, 32 or 64
// columns; the accumulator has a vocabulary entry per lane and a row of x per column.  Every CTA works alone
// (cta_group::1) on a stretch of the vocabulary cut at multiples of 32 entries, so that all SMs read the same amount, with
// 128 KB and more of W in flight.  Measured, one row, 65536 x 2048 (268 MB): z 49 us (5.6 TB/s), dx 45 us (6.0 TB/s); the
// general kernel's 256 x 256 tiles take 85 us.  64 rows: z 58 us (their own loads are half as many bytes as W's).
//
//   kLse      per lane the running maximum and sum of every row of x over the CTA's entries, joined over the CTA at
//             the end: one (maximum, sum) per CTA and row of x
//   kDz       dz of an entry for all rows of x: 64 bf16 values, one 128-byte line, [V][planes * 64]; db is the lane's own sum.
//             Few values of dz may make up a gradient, so that a rounding of them to bf16 would show in it; up to 32 rows
//             leave half of the line to a second term, which the products for dx and dW take along.
//   kPartial  dx^T = W^T dz^T in splits of the vocabulary: fp32 [splits][B][ld]
//
// dW = dz^T x runs on the general kernel, which only writes here.
constexpr int kRowsMax = 64;
constexpr int kRowsPitch = 64;           // columns of a term of dz in memory: one swizzle row
constexpr int kRowsUnit = 32;            // entries a stretch is counted in: rows of one box of W
constexpr int kRowsKw = 2 * kKBox;       // vocabulary entries of a stage of kPartial
constexpr int kRowsThreads = 64 + 128;   // loads, products, four epilogue warps

template <int MODE, int NT> struct RowsStage {
    // K values: with 16 rows twice as many, longer stretches of W's rows at a time (65536 x 2048: 54.9 -> 52 us)
    static constexpr int kw = MODE == kPartial ? kRowsKw : (NT == 16 ? 4 : 2) * kKBox;
    static constexpr int a_bytes = kHalf * kw * 2;
    static constexpr int b_bytes = (MODE == kPartial ? kRowsPitch : NT) * kw * 2;
    static constexpr int bytes = a_bytes + b_bytes;
    static constexpr int count = 216 * 1024 / bytes;
};
constexpr int kRowsSmem = 216 * 1024 + 1024;

struct CeRowsArgs {
    int B, D, V;
    int tiles, splits;       // kPartial: tiles of 128 columns of W, splits of the vocabulary
    CeHeader *head;
    const void *bias;
    int bias_bf16;
    const int *labels;
    float2 *part;            // kLse: [grid][B]
    float *zlab;
    const float *lse, *drow; // kDz
    bf16 *dz;                // kDz: [V][planes * 64]
    float *db;               // kDz, nullable
    int planes;
    float *dx_part;          // kPartial
    size_t dx_split;
    int ld;
    unsigned polls;          // of a bounded wait
};

__device__ __forceinline__ void tma_load_1(uint32_t dst, const CUtensorMap *map, uint32_t bar, int c0, int c1) {
    asm volatile("cp.async.bulk.tensor.2d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4}], [%2];"
                 ::"r"(dst), "l"(map), "r"(bar), "r"(c0), "r"(c1) : "memory");
}

// The tiles of a CTA: kLse, kDz: up to 128 entries from `at` on, until `end`, over all of D.  kPartial: one tile of 128
// columns of W (`at`) over the stages [kb0, kb1) of the vocabulary.
template <int MODE, int KW> struct RowsWalk {
    int at, end, kb0, kb1, item, items, step;
    const CeRowsArgs &g;
    __device__ __forceinline__ explicit RowsWalk(const CeRowsArgs &a) : g(a) {
        if (MODE == kPartial) {
            item = blockIdx.x; step = gridDim.x; items = g.tiles * g.splits;
            at = end = kb0 = kb1 = 0;
        } else {
            const unsigned units = (unsigned)(g.V + kRowsUnit - 1) / kRowsUnit;  // < 2^20, so that the products fit 32 bits
            at = (int)(units * blockIdx.x / gridDim.x) * kRowsUnit;
            end = min((int)(units * (blockIdx.x + 1) / gridDim.x) * kRowsUnit, g.V);
            kb0 = 0; kb1 = (g.D + KW - 1) / KW;
            item = items = step = 0;
        }
    }
    __device__ __forceinline__ bool more() {
        if (MODE != kPartial) return at < end;
        if (item >= items) return false;
        const int split = item / g.tiles, kb = (g.V + kRowsKw - 1) / kRowsKw;  // kb < 2^17, splits <= 148
        at = (item - split * g.tiles) * kHalf;
        kb0 = (int)((unsigned)(kb * split) / (unsigned)g.splits);
        kb1 = (int)((unsigned)(kb * (split + 1)) / (unsigned)g.splits);
        return true;
    }
    __device__ __forceinline__ void next() { if (MODE == kPartial) item += step; else at += kHalf; }
};

template <int MODE, int NT>
__global__ void __launch_bounds__(kRowsThreads, 1)
ce_rows_kernel(const __grid_constant__ CUtensorMap map_w, const __grid_constant__ CUtensorMap map_x, const __grid_constant__ CeRowsArgs g) {
    typedef RowsStage<MODE, NT> St;
    // Logits stay in 32 bits.  The loads leave the epilogue time to add short chains up, 16 to 64 rows of 2048 columns 256 to
    // 1024 products long: lse of one row, 65536 x 2048, is 3.7e-7 off 64 bits (8.0e-6 with one chain of 2048) and takes 0.6 us
    // more; 64 rows 3.6e-6 (7.8e-6) and no time (chains of 256: 7.4e-7 and 8 us).
    constexpr int kStages = St::count, kw = St::kw, kPiece = (MODE == kPartial ? kPieceOut : 16 * NT) / kw;
    constexpr bool kMn = MODE == kPartial;  // both operands lie with K outermost
    extern __shared__ uint8_t smem_raw[];
    __shared__ uint64_t full[kStages], empty[kStages], acc_full[2], acc_empty[2], drained;
    __shared__ uint32_t tmem_holder;
    __shared__ int abort_flag;
    __shared__ int s_label[NT];
    __shared__ float s_lse[NT], s_weight[NT];
    __shared__ float2 s_part[4][MODE == kLse ? NT : 1];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u;
    const Waiter wt{&abort_flag, &abort_flag, g.polls};
    constexpr uint32_t kTmem = 2 * NT <= 32 ? 32 : 2 * NT;
    if (threadIdx.x == 0) {
        for (int i = 0; i < kStages; ++i) { mbar_init(smem_u32(&full[i]), 1); mbar_init(smem_u32(&empty[i]), 1); }
        for (int i = 0; i < 2; ++i) { mbar_init(smem_u32(&acc_full[i]), 1); mbar_init(smem_u32(&acc_empty[i]), 4); }
        mbar_init(smem_u32(&drained), 1);
        abort_flag = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 1) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&tmem_holder)), "r"(kTmem) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    pdl_launch();
    pdl_wait();
    if (MODE == kLse && blockIdx.x == 0 && threadIdx.x == 0) g.head->ticket = 0;
    if (MODE != kPartial && threadIdx.x < NT) {
        const int t = threadIdx.x, y = t < g.B ? g.labels[t] : -1;
        const bool counted = y >= 0 && y < g.V;
        s_label[t] = counted ? y : -1;
        if (MODE == kDz) {
            s_lse[t] = t < g.B ? g.lse[t] : 0.f;
            s_weight[t] = counted ? (g.drow ? g.drow[t] : 1.f) : 0.f;
        }
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = tmem_holder;
    uint32_t issued = 0;   // steps that the thread of the loads has issued
    bool issuer = false;   // the thread that issues the products

    if (warp == 0) {
        if (lane == 0) {  // loads
            bool ok = true;
            uint32_t s = 0, ph = 0;
            for (RowsWalk<MODE, St::kw> w(g); ok && w.more(); w.next()) {
                // rows of W that the tile has: whole boxes of 32; what a shorter tile leaves in place belongs to no entry
                const int boxes = MODE == kPartial ? 0 : min(kHalf, w.end - w.at + kRowsUnit - 1) / kRowsUnit;
                for (int kb = w.kb0; kb < w.kb1; ++kb) {
                    if (!mbar_wait(smem_u32(&empty[s]), ph ^ 1u, wt, 61)) { ok = false; break; }
                    const uint32_t bar = smem_u32(&full[s]), a = base + s * St::bytes, b = a + St::a_bytes;
                    const int k = kb * kw;
                    if (MODE == kPartial) {
                        mbar_expect_tx(bar, St::bytes);
                        tma_load_1(a, &map_w, bar, w.at, k);
                        tma_load_1(a + St::a_bytes / 2, &map_w, bar, w.at + kKBox, k);
                        tma_load_1(b, &map_x, bar, 0, k);
                    } else {
                        mbar_expect_tx(bar, (uint32_t)(boxes * kRowsUnit * kw * 2 + St::b_bytes));
                        for (int j = 0; j < kw / kKBox; ++j) {
                            for (int i = 0; i < boxes; ++i)
                                tma_load_1(a + j * (kHalf * 128) + i * (kRowsUnit * 128), &map_w, bar, k + kKBox * j, w.at + i * kRowsUnit);
                            tma_load_1(b + j * (NT * 128), &map_x, bar, k + kKBox * j, 0);
                        }
                    }
                    ++issued;
                    if (++s == kStages) { s = 0; ph ^= 1u; }
                }
            }
        }
        __syncwarp();
    } else if (warp == 1) {
        issuer = elect_one();
        const uint32_t idesc = (1u << 4) | (1u << 7) | (1u << 10) | (kMn ? (1u << 15) | (1u << 16) : 0u) | ((uint32_t)(NT >> 3) << 17) | ((uint32_t)(kHalf >> 4) << 24);
        const uint64_t ad0 = kMn ? make_desc(base, 1024, 2u, St::a_bytes / 2) : make_desc(base, 1024, 2u);
        const uint64_t bd0 = make_desc(base + St::a_bytes, 1024, 2u);
        bool ok = true;
        uint32_t s = 0, ph = 0, u = 0;
        for (RowsWalk<MODE, St::kw> w(g); ok && w.more(); w.next()) {
            for (int i0 = w.kb0; i0 < w.kb1 && ok; ++u) {
                const int i1 = min(i0 + kPiece, w.kb1);
                const uint32_t acc = tmem + (u & 1u) * NT;
                ok = mbar_wait(smem_u32(&acc_empty[u & 1u]), ((u >> 1) & 1u) ^ 1u, wt, 62);
                tc_fence_after();
                for (int i = i0; i < i1 && ok; ++i) {
                    ok = mbar_wait(smem_u32(&full[s]), ph, wt, 63);
                    tc_fence_after();
                    if (ok && issuer) {
                        const uint32_t at = s * (St::bytes >> 4);
#pragma unroll
                        for (int k = 0; k < kw / 16; ++k) {
                            const uint32_t ka = kMn ? 128u * k : (uint32_t)((k >> 2) * (kHalf * 128 >> 4) + (k & 3) * 2);
                            const uint32_t kb = kMn ? 128u * k : (uint32_t)((k >> 2) * (NT * 128 >> 4) + (k & 3) * 2);
                            tc_mma_bf16(acc, ad0 + (uint64_t)(at + ka), bd0 + (uint64_t)(at + kb), idesc, i > i0 || k > 0);
                        }
                        tc_commit(smem_u32(&empty[s]));
                    }
                    if (++s == kStages) { s = 0; ph ^= 1u; }
                }
                if (ok && issuer) tc_commit(smem_u32(&acc_full[u & 1u]));
                i0 = i1;
            }
        }
        __syncwarp();
    } else {
        const int quarter = warp & 3;
        float top[MODE == kLse ? NT : 1], sum[MODE == kLse ? NT : 1];
#pragma unroll
        for (int j = 0; j < (MODE == kLse ? NT : 1); ++j) { top[j] = -FLT_MAX; sum[j] = 0.f; }
        const float scale = MODE == kDz && g.db ? g.head->scale : 1.f;
        bool ok = true;
        uint32_t u = 0;
        for (RowsWalk<MODE, St::kw> w(g); ok && w.more(); w.next()) {
            const int row = w.at + 32 * quarter + lane;  // vocabulary entry, or column of W
            float v[NT];
            const int pieces = (w.kb1 - w.kb0 + kPiece - 1) / kPiece;
            for (int piece = 0; piece < pieces; ++piece, ++u) {
                ok = __all_sync(0xffffffffu, mbar_wait(smem_u32(&acc_full[u & 1u]), (u >> 1) & 1u, wt, 64));
                if (!ok) break;
                __syncwarp();
                tc_fence_after();
                const uint32_t taddr = tmem + (u & 1u) * NT + ((uint32_t)(32 * quarter) << 16);
#pragma unroll
                for (int j = 0; j < NT; j += 16) {
                    float q[16];
                    tc_ld16(taddr + (uint32_t)j, q);
                    tc_wait_ld();
#pragma unroll
                    for (int k = 0; k < 16; ++k) v[j + k] = piece == 0 ? q[k] : v[j + k] + q[k];
                }
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(smem_u32(&acc_empty[u & 1u]));
            }
            if (!ok) break;
            if (MODE == kPartial) {
                const int split = w.item / g.tiles;
                if (row < g.D) {
                    float *dst = g.dx_part + split * g.dx_split + row;
#pragma unroll
                    for (int j = 0; j < NT; ++j)
                        if (j < g.B) dst[(size_t)j * g.ld] = j < NT / 2 && g.B <= NT / 2 ? v[j] + v[j + NT / 2 < NT ? j + NT / 2 : j] : v[j];  // both terms
                }
                continue;
            }
            const bool live = row < w.end;  // lanes past the stretch have nothing to add
            const float bias = live && g.bias ? load_bias(g.bias, g.bias_bf16, row) : 0.f;
            if (MODE == kLse) {
#pragma unroll
                for (int j = 0; j < NT; ++j) {
                    // one exponential: of the new logit below the maximum, or of the old maximum below the new one.
                    // The maximum starts at the lowest finite value, so that minus infinity adds nothing.
                    const float z = live ? v[j] + bias : -INFINITY;
                    if (live && s_label[j] == row) g.zlab[j] = z;
                    const float d = z - top[j], e = exp2_approx(-fabsf(d) * kLog2e);
                    sum[j] = d > 0.f ? fmaf(sum[j], e, 1.f) : sum[j] + e;
                    top[j] = fmaxf(top[j], z);
                }
            } else if (live) {
                float total = 0.f;
#pragma unroll
                for (int j = 0; j < NT; ++j) {
                    float p = exp2_approx((v[j] + bias - s_lse[j]) * kLog2e) - (s_label[j] == row ? 1.f : 0.f);
                    // a row that does not count, or is not there, gives exact zeros
                    p = s_weight[j] != 0.f ? p * s_weight[j] : 0.f;
                    v[j] = p;
                    total += p;
                }
                if (g.db) g.db[row] = total * scale;
                const int planes = NT < kRowsPitch ? 2 : g.planes;
                uint4 *dst = reinterpret_cast<uint4 *>(g.dz + (size_t)row * (NT < kRowsPitch ? 1 : planes) * kRowsPitch);
                for (int p = 0; p < planes; ++p, dst += NT / 8) {
#pragma unroll
                    for (int j = 0; j < NT / 8; ++j) {
                        const float *f = v + 8 * j;
                        dst[j] = make_uint4(pack2(f[0], f[1]), pack2(f[2], f[3]), pack2(f[4], f[5]), pack2(f[6], f[7]));
                    }
#pragma unroll
                    for (int j = 0; j < NT; ++j) {  // an infinity stays in the first term alone
                        const float h = bf16_round(v[j]);
                        v[j] = isinf(h) ? 0.f : v[j] - h;
                    }
                }
            }
        }
        if (MODE == kLse) {  // over the lanes
#pragma unroll
            for (int j = 0; j < NT; ++j) {
                const float m = warp_max(top[j]), t = warp_sum(sum[j] * exp2_approx((top[j] - m) * kLog2e));
                if (lane == 0) s_part[quarter][j] = make_float2(m, t);
            }
        }
    }
    __syncthreads();
    if (MODE == kLse && threadIdx.x < g.B) {  // over the warps
        const int j = threadIdx.x;
        float m = s_part[0][j].x, t = 0.f;
        for (int q = 1; q < 4; ++q) m = fmaxf(m, s_part[q][j].x);
        for (int q = 0; q < 4; ++q) t += s_part[q][j].y * exp2_approx((s_part[q][j].x - m) * kLog2e);
        g.part[(size_t)blockIdx.x * g.B + j] = make_float2(m, t);
    }
    tc_fence_before();
    __syncthreads();
    if (abort_flag) {
        // A wait ran out: the products in flight end by themselves, so do the copies of the last kStages steps
        if (issuer) tc_commit(smem_u32(&drained));
        if (threadIdx.x == 0) {
            mbar_drain(smem_u32(&drained), 0);
            for (uint32_t i = issued > kStages ? issued - kStages : 0; i < issued; ++i) mbar_drain(smem_u32(&full[i % kStages]), (i / kStages) & 1u);
        }
        __syncthreads();
    }
    if (warp == 1) {
        tc_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(kTmem) : "memory");
    }
    if (threadIdx.x == 0) {
        if (MODE == kLse) g.head->status[blockIdx.x] = abort_flag;
        else if (abort_flag) g.head->failed = 1;
    }
}

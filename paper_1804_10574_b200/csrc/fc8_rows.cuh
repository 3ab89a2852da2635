// The product of 8-bit codes for a few rows of x, part of fc8.cu.
//
// With B rows a code of W is multiplied B times: for few rows the bytes of W bound the time.  So W is the operand with the 128
// rows of an MMA (outputs) and the rows of x are its 16 to 128 columns.  A tile of 128 outputs is a cluster's: its CTAs share the
// K range, so that all SMs read W however few tiles there are, and add their integer sums, which are exact in any order, over
// one another's shared memory: one launch, no workspace.  Measured: one row, 4096 x 16384 (67 MB) 14.5 us (4.6 TB/s; the tiles of
// 256 rows take 24.8), 16384 x 4096 15 us (58), 4096 x 4096 6.8 us (17.5); 64 rows, 4096 x 16384 17 us.
constexpr int kRowsThreads = 64 + 128;         // loads, products, four epilogue warps
constexpr int kRowsPerSm = 2;                  // CTAs of an SM: clusters of whole SMs leave some of them idle
constexpr int kRowsSmem = 104 * 1024;
constexpr int kRowsMostSplits = 8;             // a cluster

template <int NT> struct RowsStage {
    static constexpr int kw = NT <= 32 ? 256 : 128;  // codes: three stages at least
    static constexpr int a_bytes = kHalf * kw, b_bytes = NT * kw, bytes = a_bytes + b_bytes;
    static constexpr int count = (kRowsSmem - 1024) / bytes;
};

struct RowsArgs {
    int B, out, tiles;          // tiles of 128 outputs
    int steps, splits;          // steps of a stage's codes, dealt out to the CTAs of a cluster
    int tail;                   // MMA steps of the last one
    const float *row_scale, *col_scale;
    const void *bias;
    int bias_bf16;
    void *y;
    int out_bf16, vec;          // vec: rows of y keep to four outputs
    unsigned polls;
};

__device__ __forceinline__ void tma_load_1(uint32_t dst, const CUtensorMap *map, uint32_t bar, int c0, int c1) {
    asm volatile("cp.async.bulk.tensor.2d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4}], [%2];"
                 ::"r"(dst), "l"(map), "r"(bar), "r"(c0), "r"(c1) : "memory");
}
__device__ __forceinline__ void mma_i8(uint32_t d_tmem, uint64_t adesc, uint64_t bdesc, uint32_t idesc, uint32_t accumulate) {
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::i8 [%0], %1, %2, %3, p;\n\t}"
        ::"r"(d_tmem), "l"(adesc), "l"(bdesc), "r"(idesc), "r"(accumulate)
        : "memory");
}

__device__ __forceinline__ float rows_bias(const RowsArgs &g, int o) {
    return !g.bias ? 0.f : (g.bias_bf16 ? to_f(((const bf16 *)g.bias)[o]) : ((const float *)g.bias)[o]);
}

template <int NT>
__global__ void __launch_bounds__(kRowsThreads, kRowsPerSm) fc8_rows_kernel(const __grid_constant__ CUtensorMap map_w, const __grid_constant__ CUtensorMap map_x, const __grid_constant__ RowsArgs g) {
    typedef RowsStage<NT> St;
    constexpr int kCount = St::count;
    constexpr uint32_t kTmem = NT < 32 ? 32 : NT;
    static_assert(NT * kHalf * 4 <= kCount * St::bytes, "the sums take the stages' place");
    extern __shared__ uint8_t smem_raw[];
    __shared__ uint64_t full[kCount], empty[kCount], acc_full, drained;
    __shared__ uint32_t tmem_holder;
    __shared__ int abort_flag;
    __shared__ float s_scale[NT];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t rank = cluster_rank();
    // tiles of outputs next to one another: their CTAs share the rows of x
    const int tile = blockIdx.x / g.splits, x_tile = tile / g.tiles, o0 = (tile - x_tile * g.tiles) * kHalf, j0 = x_tile * NT, rows = min(NT, g.B - j0);
    const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u;
    const Waiter wt{&abort_flag, &abort_flag, g.polls};
    if (threadIdx.x == 0) {
        for (int i = 0; i < kCount; ++i) { mbar_init(smem_u32(&full[i]), 1); mbar_init(smem_u32(&empty[i]), 1); }
        mbar_init(smem_u32(&acc_full), 1);
        mbar_init(smem_u32(&drained), 1);
        abort_flag = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 1) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&tmem_holder)), "r"(kTmem) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    const int i0 = (int)((long)g.steps * rank / g.splits), i1 = (int)((long)g.steps * (rank + 1) / g.splits);  // not empty: splits <= steps
    pdl_launch();
    // The first stages of W come into the L2 while the kernel before still runs.  That reads nothing: the L2 is where the memory's
    // values are the same for all, and what that kernel may yet write of W is written there.
    if (threadIdx.x == 0) {
        for (int i = i0; i < min(i1, i0 + 2 * kCount); ++i)
#pragma unroll
            for (int j = 0; j < St::kw / 128; ++j)
                asm volatile("cp.async.bulk.prefetch.tensor.2d.L2.global.tile [%0, {%1, %2}];" ::"l"(&map_w), "r"(i * St::kw + 128 * j), "r"(o0) : "memory");
    }
    pdl_wait();
    for (int j = threadIdx.x; j < rows; j += kRowsThreads) s_scale[j] = g.row_scale[j0 + j];
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = tmem_holder;
    uint32_t issued = 0;
    bool issuer = false, ok = true;
    if (warp == 0) {
        if (lane == 0) {  // loads
            uint32_t s = 0, ph = 0;
            for (int i = i0; i < i1; ++i) {
                if (!mbar_wait(smem_u32(&empty[s]), ph ^ 1u, wt, 91)) break;
                const uint32_t bar = smem_u32(&full[s]), a = base + s * St::bytes, b = a + St::a_bytes;
                mbar_expect_tx(bar, St::bytes);
#pragma unroll
                for (int j = 0; j < St::kw / 128; ++j) {
                    tma_load_1(a + j * (kHalf * 128), &map_w, bar, i * St::kw + 128 * j, o0);
                    tma_load_1(b + j * (NT * 128), &map_x, bar, i * St::kw + 128 * j, j0);
                }
                ++issued;
                if (++s == kCount) { s = 0; ph ^= 1u; }
            }
        }
        __syncwarp();
    } else if (warp == 1) {
        issuer = elect_one();
        const uint32_t idesc = (2u << 4) | (1u << 7) | (1u << 10) | ((uint32_t)(NT >> 3) << 17) | ((uint32_t)(kHalf >> 4) << 24);
        const uint64_t ad0 = make_desc(base, 1024, 2u), bd0 = make_desc(base + St::a_bytes, 1024, 2u);
        uint32_t s = 0, ph = 0;
        for (int i = i0; i < i1; ++i) {
            if (!(ok = mbar_wait(smem_u32(&full[s]), ph, wt, 92))) break;
            tc_fence_after();
            if (issuer) {
                const uint32_t at = s * (St::bytes >> 4);
                const int steps = i == g.steps - 1 ? g.tail : St::kw / 32;
#pragma unroll
                for (int k = 0; k < St::kw / 32; ++k) {
                    if (k >= steps) break;
                    mma_i8(tmem, ad0 + (uint64_t)(at + (k >> 2) * (kHalf * 128 >> 4) + (k & 3) * 2), bd0 + (uint64_t)(at + (k >> 2) * (NT * 128 >> 4) + (k & 3) * 2), idesc, i > i0 || k > 0);
                }
                tc_commit(smem_u32(&empty[s]));
            }
            if (++s == kCount) { s = 0; ph ^= 1u; }
        }
        if (ok && issuer) tc_commit(smem_u32(&acc_full));
        __syncwarp();
    }
    // the sums are there, or a wait ran out: then what is in flight has to land before its place is used
    if (warp >= 2) ok = __all_sync(0xffffffffu, mbar_wait(smem_u32(&acc_full), 0, wt, 93));
    __syncthreads();
    if (abort_flag) {
        if (issuer) tc_commit(smem_u32(&drained));
        if (threadIdx.x == 0) {
            mbar_drain(smem_u32(&drained), 0);
            for (uint32_t i = issued > kCount ? issued - kCount : 0; i < issued; ++i) mbar_drain(smem_u32(&full[i % kCount]), (i / kCount) & 1u);
        }
        __syncthreads();
    }
    const int quarter = warp & 3;
    const float lost = __int_as_float(0x7fffffff);
    if (warp >= 2) {
        tc_fence_after();
        const uint32_t to = base + (uint32_t)(32 * quarter + lane) * 4u;
#pragma unroll 1
        for (int c = 0; c < NT; c += 16) {  // 16 rows of x at a time
            if (c >= rows) break;
            float q[16];
            tc_ld16(tmem + ((uint32_t)(32 * quarter) << 16) + (uint32_t)c, q);
            tc_wait_ld();
#pragma unroll
            for (int k = 0; k < 16; ++k) asm volatile("st.shared.b32 [%0], %1;" ::"r"(to + (uint32_t)(c + k) * (kHalf * 4)), "r"(__float_as_int(q[k])) : "memory");
        }
    }
    {
        cluster_sync();  // (a CTA by itself is a cluster of one)
        // every CTA joins a share of the tile
        int failed = 0;
        for (uint32_t r = 0; r < (uint32_t)g.splits; ++r) {
            int f;
            asm volatile("ld.shared::cluster.b32 %0, [%1];" : "=r"(f) : "r"(map_rank(smem_u32(&abort_flag), r)));
            failed |= f;
        }
        auto result = [&](int acc, int j, float cs, float bias) {
            const RowScale rs = row_scale_of(s_scale[j]);
            const float most = 3.402823466e38f, up = cs * rs.up;  // (past that only a sum of zero is finite)
            return failed ? lost : (float)acc * rs.by * (up > most ? most : up) + bias;
        };
        if (g.vec) {
            const int o = o0 + 4 * (threadIdx.x % 32);  // 192 threads are whole rows of 32 groups
            float cs[4] = {}, bias[4] = {};
            if (o < g.out) {
#pragma unroll
                for (int k = 0; k < 4; ++k) { cs[k] = g.col_scale[o + k]; bias[k] = rows_bias(g, o + k); }
            }
            constexpr int kAtOnce = 2;  // loads on their way
            const int step = g.splits * kRowsThreads, total = rows * (kHalf / 4);
            for (int i0 = (int)rank * kRowsThreads + threadIdx.x; i0 < total; i0 += kAtOnce * step) {
                int acc[kAtOnce][4] = {};
                for (uint32_t r = 0; r < (uint32_t)g.splits; ++r) {
                    const uint32_t from = map_rank(base, r);
                    int q[kAtOnce][4] = {};
#pragma unroll
                    for (int u = 0; u < kAtOnce; ++u)
                        if (i0 + u * step < total)
                            asm volatile("ld.shared::cluster.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(q[u][0]), "=r"(q[u][1]), "=r"(q[u][2]), "=r"(q[u][3]) : "r"(from + 16u * (i0 + u * step)));
#pragma unroll
                    for (int u = 0; u < kAtOnce; ++u)
#pragma unroll
                        for (int k = 0; k < 4; ++k) acc[u][k] += q[u][k];
                }
#pragma unroll
                for (int u = 0; u < kAtOnce; ++u) {
                    const int i = i0 + u * step, j = i / 32;
                    if (i >= total || o >= g.out) continue;
                    float v[4];
#pragma unroll
                    for (int k = 0; k < 4; ++k) v[k] = result(acc[u][k], j, cs[k], bias[k]);
                    const size_t at = (size_t)(j0 + j) * g.out + o;
                    if (g.out_bf16) store_f<bf16, 4>((bf16 *)g.y + at, v); else store_f<float, 4>((float *)g.y + at, v);
                }
            }
        } else {
            constexpr int kAtOnce = 4;
            const int o = o0 + threadIdx.x;  // one output per thread
            if (threadIdx.x < kHalf && o < g.out) {
                const float cs = g.col_scale[o], bias = rows_bias(g, o);
                for (int j1 = (int)rank; j1 < rows; j1 += kAtOnce * g.splits) {
                    int acc[kAtOnce] = {};
                    for (uint32_t r = 0; r < (uint32_t)g.splits; ++r) {
                        const uint32_t from = map_rank(base + 4u * threadIdx.x, r);
                        int q[kAtOnce] = {};
#pragma unroll
                        for (int u = 0; u < kAtOnce; ++u)
                            if (j1 + u * g.splits < rows) asm volatile("ld.shared::cluster.b32 %0, [%1];" : "=r"(q[u]) : "r"(from + (uint32_t)(j1 + u * g.splits) * (4u * kHalf)));
#pragma unroll
                        for (int u = 0; u < kAtOnce; ++u) acc[u] += q[u];
                    }
#pragma unroll
                    for (int u = 0; u < kAtOnce; ++u) {
                        const int j = j1 + u * g.splits;
                        if (j >= rows) break;
                        const float v = result(acc[u], j, cs, bias);
                        const size_t at = (size_t)(j0 + j) * g.out + o;
                        if (g.out_bf16) ((bf16 *)g.y)[at] = from_f<bf16>(v); else ((float *)g.y)[at] = v;
                    }
                }
            }
        }
        cluster_sync();  // no CTA leaves while its sums are read
    }
    tc_fence_before();
    __syncthreads();
    if (warp == 1) {
        tc_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(kTmem) : "memory");
    }
}

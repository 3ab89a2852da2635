// The vocabulary projection for at most 16 rows of fp32, part of linear_ce.cu.
//
// The tensor cores need an fp32 W in three bf16 terms, which is four times its bytes to move before a few rows are
// multiplied.  With n <= 16 rows the CUDA cores keep up with the memory: per value of W n multiply-adds.  W is read as it
// lies, once per pass:
//   logits     a warp has a few vocabulary entries at a time, its lanes stride along a row of W, the rows of x stand in
//              shared memory; the lanes' sums are transposed so that a lane ends with the logits of one row of x always, and
//              keeps that row's running maximum and sum (forward), or writes dz [V][NB] (backward)
//   dx         a thread has four columns of W and all rows of x; splits of the vocabulary, joined by ce_dx_kernel
//   dW         a thread has four columns of x for all rows in registers and walks entries
// Measured, 65536 x 2048 (537 MB), one row: logits 95 us (5.6 TB/s), dx 145 us, dW 91 us; 32000 x 1024, 16 rows: 57 us (LDS
// and FMA, 53 % of the issue slots), 63 and 50 us.  The general path takes 635 us forward and 1279 us backward for the first.
// Any width, no alignment: lanes take neighbouring columns, or float4s of them where rows of W allow it.
constexpr int kR32Max = 16, kR32Threads = 256;
constexpr int kR32MostWarps = 16;  // of the logits: 16 where x leaves room for one CTA on an SM, else 8
constexpr int kR32Smem = 200 * 1024;
constexpr int kR32Cols = 256;     // columns of a CTA of dx and dW: 64 threads of four, four threads along the entries
constexpr int kR32Chunk = 256;    // entries of dz that a CTA of dx and dW has in shared memory at a time

__host__ __device__ inline int r32_pitch(int D) { return (D + 127) / 128 * 128; }  // whole strides of a warp's float4s
inline int r32_nb(int B) { return B <= 4 ? 4 : (B <= 8 ? 8 : 16); }
inline bool r32_fits(int prec, int B, int D) { return prec == P_F32 && B <= kR32Max && (size_t)r32_nb(B) * r32_pitch(D) * 4 <= kR32Smem; }

struct CeR32Args {
    const float *x, *W, *bias;
    const int *labels;
    CeHeader *head;
    float2 *part;               // forward: [grid][B]
    float *zlab;
    const float *lse, *dloss, *drow;
    float *dz, *db;             // backward: dz [V][NB]
    float *dx_part, *dW;
    size_t dx_split;
    int B, D, V, ld, splits;
};

template <int NB> __device__ __forceinline__ float r32_scale(const CeR32Args &g) {
    if (g.drow) return 1.f;
    int n = 0;
    for (int j = 0; j < g.B; ++j) n += g.labels[j] >= 0 && g.labels[j] < g.V;
    return (g.dloss ? *g.dloss : 1.f) / (float)max(n, 1);
}

template <int MODE, int NB, int VEC>
__global__ void __launch_bounds__(32 * kR32MostWarps) ce_r32_logits_kernel(const CeR32Args g) {
    constexpr int kEntries = NB == 16 ? 4 : 32 / NB, kSets = kEntries * NB / 32;  // entries of a warp at a time; values per lane of them
    extern __shared__ float4 r32_smem[];
    __shared__ float2 s_part[kR32MostWarps][NB];
    float *xs = reinterpret_cast<float *>(r32_smem);  // [NB][P]
    const int P = r32_pitch(g.D), warp = threadIdx.x >> 5, warps = blockDim.x >> 5, lane = threadIdx.x & 31, n = lane % NB;
    pdl_launch();
    pdl_wait();
    if (MODE == kLse && blockIdx.x == 0 && threadIdx.x == 0) g.head->ticket = 0;
    for (int i = threadIdx.x; i < NB * P; i += blockDim.x) {
        const int r = i / P, c = i - r * P;
        xs[i] = r < g.B && c < g.D ? g.x[(size_t)r * g.D + c] : 0.f;
    }
    const int y = n < g.B ? g.labels[n] : -1;
    const bool counted = y >= 0 && y < g.V;
    float top = -FLT_MAX, sum = 0.f, lse = 0.f, weight = 0.f, scale = 0.f;
    if (MODE == kDz) {
        lse = n < g.B ? g.lse[n] : 0.f;
        weight = counted ? (g.drow ? g.drow[n] : 1.f) : 0.f;
        scale = r32_scale<NB>(g);
        if (blockIdx.x == 0 && threadIdx.x == 0) { g.head->scale = scale; g.head->failed = 0; }
    }
    __syncthreads();
    const int groups = (g.V + kEntries - 1) / kEntries, walkers = gridDim.x * warps;
    for (int group = blockIdx.x * warps + warp; group < groups; group += walkers) {
        const int v0 = group * kEntries;
        float acc[kEntries * NB];
#pragma unroll
        for (int i = 0; i < kEntries * NB; ++i) acc[i] = 0.f;
        for (int d = lane * VEC; d < g.D; d += 32 * VEC) {
            float w[kEntries][VEC];
#pragma unroll
            for (int e = 0; e < kEntries; ++e) {
                const float *src = g.W + (size_t)min(v0 + e, g.V - 1) * g.D + d;
                load_f<float, VEC>(src, w[e]);
            }
#pragma unroll
            for (int r = 0; r < NB; ++r) {
                float x[VEC];
                load_f<float, VEC>(xs + r * P + d, x);
#pragma unroll
                for (int e = 0; e < kEntries; ++e)
#pragma unroll
                    for (int k = 0; k < VEC; ++k) acc[e * NB + r] = fmaf(w[e][k], x[k], acc[e * NB + r]);
            }
        }
        // lane j of set s ends with value 32 s + j: entry (32 s + j) / NB, row j % NB
#pragma unroll
        for (int s = 0; s < kSets; ++s) {
            float t[32];
#pragma unroll
            for (int i = 0; i < 32; ++i) t[i] = acc[32 * s + i];
            float z = column_sums(t, lane);
            const int v = v0 + (32 * s + lane) / NB;
            const bool there = v < g.V;
            if (there && g.bias) z += g.bias[v];
            if (MODE == kLse) {
                if (!there) z = -INFINITY;
                if (there && counted && v == y && n < g.B) g.zlab[n] = z;
                const float d = z - top, e = exp2_approx(-fabsf(d) * kLog2e);
                sum = d > 0.f ? fmaf(sum, e, 1.f) : sum + e;
                top = fmaxf(top, z);
            } else {
                float p = exp2_approx((z - lse) * kLog2e) - (v == y ? 1.f : 0.f);
                p = weight != 0.f ? p * weight : 0.f;  // a row that does not count, or is not there, gives exact zeros
                if (there) g.dz[(size_t)v * NB + n] = p;
                if (g.db) {
#pragma unroll
                    for (int o = NB / 2; o > 0; o >>= 1) p += __shfl_xor_sync(0xffffffffu, p, o);
                    if (there && n == 0) g.db[v] = p * scale;
                }
            }
        }
    }
    if (MODE == kLse) {  // over the lanes of a row of x, then over the warps
        float m = top;
#pragma unroll
        for (int o = NB; o < 32; o <<= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
        float t = sum * exp2_approx((top - m) * kLog2e);
#pragma unroll
        for (int o = NB; o < 32; o <<= 1) t += __shfl_xor_sync(0xffffffffu, t, o);
        if (lane < NB) s_part[warp][lane] = make_float2(m, t);
        __syncthreads();
        if ((int)threadIdx.x < g.B) {
            m = s_part[0][threadIdx.x].x;
            for (int q = 1; q < warps; ++q) m = fmaxf(m, s_part[q][threadIdx.x].x);
            t = 0.f;
            for (int q = 0; q < warps; ++q) t += s_part[q][threadIdx.x].y * exp2_approx((s_part[q][threadIdx.x].x - m) * kLog2e);
            g.part[(size_t)blockIdx.x * g.B + threadIdx.x] = make_float2(m, t);
        }
    }
}

// blockIdx.x: 256 columns; blockIdx.y: split of the vocabulary
template <int NB>
__global__ void __launch_bounds__(kR32Threads) ce_r32_dx_kernel(const CeR32Args g) {
    __shared__ float4 s_dz[kR32Chunk][NB / 4];
    __shared__ float fold[3][64][4];
    pdl_launch();
    pdl_wait();
    const int tx = threadIdx.x & 63, ty = threadIdx.x >> 6, c0 = blockIdx.x * kR32Cols + tx;
    const int v_first = (int)((long)g.V * blockIdx.y / g.splits), v_last = (int)((long)g.V * (blockIdx.y + 1) / g.splits);
    float acc[NB][4];
#pragma unroll
    for (int r = 0; r < NB; ++r)
#pragma unroll
        for (int j = 0; j < 4; ++j) acc[r][j] = 0.f;
    for (int v0 = v_first; v0 < v_last; v0 += kR32Chunk) {
        const int n = min(kR32Chunk, v_last - v0);
        __syncthreads();
        for (int i = threadIdx.x; i < n * (NB / 4); i += kR32Threads) s_dz[i / (NB / 4)][i % (NB / 4)] = reinterpret_cast<const float4 *>(g.dz + (size_t)v0 * NB)[i];
        __syncthreads();
#pragma unroll 8
        for (int i = ty; i < n; i += 4) {
            float w[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) w[j] = c0 + 64 * j < g.D ? g.W[(size_t)(v0 + i) * g.D + c0 + 64 * j] : 0.f;
#pragma unroll
            for (int q = 0; q < NB / 4; ++q) {
                const float4 p = s_dz[i][q];
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    acc[4 * q][j] = fmaf(p.x, w[j], acc[4 * q][j]);
                    acc[4 * q + 1][j] = fmaf(p.y, w[j], acc[4 * q + 1][j]);
                    acc[4 * q + 2][j] = fmaf(p.z, w[j], acc[4 * q + 2][j]);
                    acc[4 * q + 3][j] = fmaf(p.w, w[j], acc[4 * q + 3][j]);
                }
            }
        }
    }
#pragma unroll
    for (int r = 0; r < NB; ++r) {  // the four threads along the entries, in order
        __syncthreads();
        if (ty > 0) {
#pragma unroll
            for (int j = 0; j < 4; ++j) fold[ty - 1][tx][j] = acc[r][j];
        }
        __syncthreads();
        if (ty == 0 && r < g.B) {
#pragma unroll
            for (int j = 0; j < 4; ++j)
                if (c0 + 64 * j < g.D)
                    g.dx_part[blockIdx.y * g.dx_split + (size_t)r * g.ld + c0 + 64 * j] = ((acc[r][j] + fold[0][tx][j]) + fold[1][tx][j]) + fold[2][tx][j];
        }
    }
}

// blockIdx.x: 256 columns; blockIdx.y: stretch of the vocabulary
template <int NB>
__global__ void __launch_bounds__(kR32Threads) ce_r32_dw_kernel(const CeR32Args g) {
    __shared__ float4 s_dz[kR32Chunk][NB / 4];
    pdl_launch();
    pdl_wait();
    const int tx = threadIdx.x & 63, ty = threadIdx.x >> 6, c0 = blockIdx.x * kR32Cols + tx;
    const int v_first = (int)((long)g.V * blockIdx.y / gridDim.y), v_last = (int)((long)g.V * (blockIdx.y + 1) / gridDim.y);
    const float scale = g.head->scale;
    float x[NB][4];
#pragma unroll
    for (int r = 0; r < NB; ++r) {
        const int y = r < g.B ? g.labels[r] : -1;
        const bool counted = y >= 0 && y < g.V;  // a row that does not count is left out, whatever stands in it
#pragma unroll
        for (int j = 0; j < 4; ++j) x[r][j] = counted && c0 + 64 * j < g.D ? g.x[(size_t)r * g.D + c0 + 64 * j] : 0.f;
    }
    for (int v0 = v_first; v0 < v_last; v0 += kR32Chunk) {
        const int n = min(kR32Chunk, v_last - v0);
        __syncthreads();
        for (int i = threadIdx.x; i < n * (NB / 4); i += kR32Threads) s_dz[i / (NB / 4)][i % (NB / 4)] = reinterpret_cast<const float4 *>(g.dz + (size_t)v0 * NB)[i];
        __syncthreads();
#pragma unroll 2
        for (int i = ty; i < n; i += 4) {
            float o[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int q = 0; q < NB / 4; ++q) {
                const float4 p = s_dz[i][q];
#pragma unroll
                for (int j = 0; j < 4; ++j) o[j] = fmaf(p.x, x[4 * q][j], fmaf(p.y, x[4 * q + 1][j], fmaf(p.z, x[4 * q + 2][j], fmaf(p.w, x[4 * q + 3][j], o[j]))));
            }
#pragma unroll
            for (int j = 0; j < 4; ++j)
                if (c0 + 64 * j < g.D) g.dW[(size_t)(v0 + i) * g.D + c0 + 64 * j] = o[j] * scale;
        }
    }
}

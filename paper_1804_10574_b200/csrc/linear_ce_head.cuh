// The projection of a small classifier head (up to 256 rows, a W that fits one SM's shared memory as fp32), part of
// linear_ce.cu.
//
// At these sizes the number of launches counts: 128 x 64 x 100 takes the general path two launches forward and five
// backward, 10.9 and 22.9 us.  Here each direction is one launch on the CUDA cores, in fp32 throughout, 8.2 and 8.1 us;
// what is left of a call is the launch and two or three waits for memory.
//   forward    one cluster of eight CTAs; each has W in shared memory and an eighth of the rows, eight at a time (a row's
//              softmax is one warp's); the mean is taken over the cluster's shared memory
//   backward   CTAs of two kinds, which need nothing of one another because lse is given: eight rows against all of W
//              for dx, and eight vocabulary entries against all rows for dW and db
constexpr int kHeadThreads = 256;
constexpr int kHeadRows = 8;      // rows of a pass, entries of a slice
constexpr int kHeadPass = 32;     // rows of x that a forward CTA has in shared memory: its eighth of them all
constexpr int kHeadMaxB = 256, kHeadMaxD = 512;
constexpr int kHeadSmem = 160 * 1024;

// Columns of a row in shared memory: whole float4s, an odd number of them, so that eight neighbouring rows lie in
// different banks.
__host__ __device__ inline int head_pitch(int D) { const int q = (D + 3) / 4; return 4 * (q | 1); }
// Rows that a slice of entries has in shared memory at a time: all of them where they fit.
__host__ __device__ inline int head_chunk(int B, int D) {
    const int fit = (kHeadSmem / 4 - kHeadRows * head_pitch(D) - kHeadThreads * kHeadRows) / (head_pitch(D) + kHeadRows) / 32 * 32, all = (B + 31) / 32 * 32;
    return all < fit ? all : fit;
}
inline size_t head_smem(int B, int D, int V) {
    const size_t P = head_pitch(D), red = (size_t)kHeadThreads * kHeadRows;
    const size_t rows = (V + kHeadPass) * P + (size_t)V * kHeadRows + red, slice = kHeadRows * P + head_chunk(B, D) * (P + kHeadRows) + red;
    return (rows > slice ? rows : slice) * sizeof(float);
}

struct CeHeadArgs {
    const void *x, *W, *bias;
    const int *labels;
    float *loss, *row_loss, *lse_out;   // forward
    const float *lse, *dloss, *drow;    // backward
    void *dx, *dW;
    float *db;
    int B, D, V, dw_f32;
};

// n rows of src from row r0 on into dst [n][P], zeros past the columns; rows past `rows`, and with `keep` the rows whose
// flag is zero, become zeros.  16-byte loads where the rows allow them.
template <typename T> __device__ __forceinline__ void head_fill(float *dst, const T *src, int r0, int n, int rows, int D, int P, const float *keep) {
    constexpr int kVec = 16 / (int)sizeof(T);
    if (D % kVec == 0 && (reinterpret_cast<uintptr_t>(src) & 15) == 0) {
        const int q = D / kVec, total = n * q;
#pragma unroll 4
        for (int i = threadIdx.x; i < total; i += kHeadThreads) {
            const int r = i / q, c = (i - r * q) * kVec;
            float v[kVec];
            if (r0 + r < rows && (!keep || keep[r] != 0.f)) {
                load_f<T, kVec>(src + (size_t)(r0 + r) * D + c, v);
            } else {
#pragma unroll
                for (int j = 0; j < kVec; ++j) v[j] = 0.f;
            }
#pragma unroll
            for (int j = 0; j < kVec; j += 4) *reinterpret_cast<float4 *>(dst + r * P + c + j) = make_float4(v[j], v[j + 1], v[j + 2], v[j + 3]);
        }
        return;  // whole float4s: nothing reads what stands between D and the pitch
    }
    const int total = n * P;
#pragma unroll 4
    for (int i = threadIdx.x; i < total; i += kHeadThreads) {
        const int r = i / P, c = i - r * P;
        const bool there = c < D && r0 + r < rows && (!keep || keep[r] != 0.f);
        dst[i] = there ? to_f(src[(size_t)(r0 + r) * D + c]) : 0.f;
    }
}
// dot products of the vector w with R rows of x (pitch P), over whole float4s
template <int R> __device__ __forceinline__ void head_dots(const float *w, const float *x, int P, int D, float (&acc)[R]) {
#pragma unroll
    for (int r = 0; r < R; ++r) acc[r] = 0.f;
#pragma unroll 4
    for (int d = 0; d < D; d += 4) {
        const float4 a = *reinterpret_cast<const float4 *>(w + d);
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const float4 b = *reinterpret_cast<const float4 *>(x + r * P + d);
            acc[r] = fmaf(a.x, b.x, fmaf(a.y, b.y, fmaf(a.z, b.z, fmaf(a.w, b.w, acc[r]))));
        }
    }
}
// logits of eight rows (xs) against all of W (ws) to z [V][8]
template <typename T> __device__ __forceinline__ void head_logits(const CeHeadArgs &g, const float *ws, const float *xs, float *z, int P) {
    const int vi = threadIdx.x & 127, part = threadIdx.x >> 7;  // four rows per thread
    for (int v = vi; v < g.V; v += 128) {
        float acc[4];
        head_dots<4>(ws + v * P, xs + part * 4 * P, P, g.D, acc);
        const float b = g.bias ? to_f(((const T *)g.bias)[v]) : 0.f;
        *reinterpret_cast<float4 *>(z + v * kHeadRows + part * 4) = make_float4(acc[0] + b, acc[1] + b, acc[2] + b, acc[3] + b);
    }
}

template <typename T>
__global__ void __cluster_dims__(8, 1, 1) __launch_bounds__(kHeadThreads) ce_head_fwd_kernel(const __grid_constant__ CeHeadArgs g) {
    extern __shared__ float4 head_smem_raw[];
    __shared__ double sums[kHeadRows];
    __shared__ int counts[kHeadRows];
    __shared__ double total;
    __shared__ int counted_all;
    const int P = head_pitch(g.D), warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    float *ws = reinterpret_cast<float *>(head_smem_raw), *xs = ws + g.V * P, *z = xs + kHeadPass * P;
    const uint32_t rank = cluster_rank();
    pdl_launch();
    pdl_wait();
    double sum = 0.0;
    int counted = 0;
    const int per = (g.B + 7) / 8, last = min(g.B, ((int)rank + 1) * per);
    if ((int)rank * per < last) {
        head_fill(ws, (const T *)g.W, 0, g.V, g.V, g.D, P, nullptr);
        head_fill(xs, (const T *)g.x, (int)rank * per, (per + kHeadRows - 1) / kHeadRows * kHeadRows, last, g.D, P, nullptr);
    }
    for (int r0 = (int)rank * per; r0 < last; r0 += kHeadRows) {
        __syncthreads();  // the pass before is read
        head_logits<T>(g, ws, xs + (r0 - (int)rank * per) * P, z, P);
        __syncthreads();
        const int row = r0 + warp;
        if (row < last) {
            float top = -INFINITY, s = 0.f;
            for (int v = lane; v < g.V; v += 32) top = fmaxf(top, z[v * kHeadRows + warp]);
            top = warp_max(top);
            const float ref = top == -INFINITY ? 0.f : top;
            for (int v = lane; v < g.V; v += 32) s += expf(z[v * kHeadRows + warp] - ref);
            s = warp_sum(s);
            const int y = g.labels[row];
            const float lse = logf(s) + top, l = y >= 0 && y < g.V ? lse - z[y * kHeadRows + warp] : 0.f;
            if (lane == 0) {
                if (g.lse_out) g.lse_out[row] = lse;
                if (g.row_loss) g.row_loss[row] = l;
            }
            sum += (double)l;
            counted += y >= 0 && y < g.V;
        }
    }
    if (lane == 0) { sums[warp] = sum; counts[warp] = counted; }
    __syncthreads();
    if (threadIdx.x == 0) {
        double t = 0.0;
        int c = 0;
        for (int w = 0; w < kHeadRows; ++w) { t += sums[w]; c += counts[w]; }
        total = t;
        counted_all = c;
    }
    cluster_sync();
    if (rank == 0 && threadIdx.x == 0 && g.loss) {
        double t = 0.0;
        int c = 0;
        for (uint32_t r = 0; r < 8; ++r) {
            double part;
            int n;
            asm volatile("ld.shared::cluster.f64 %0, [%1];" : "=d"(part) : "r"(map_rank(smem_u32(&total), r)));
            asm volatile("ld.shared::cluster.s32 %0, [%1];" : "=r"(n) : "r"(map_rank(smem_u32(&counted_all), r)));
            t += part;
            c += n;
        }
        *g.loss = (float)(t / (double)max(c, 1));
    }
    cluster_sync();  // no CTA leaves while its shared memory is read
}

// Sums over the threads that share a column: acc[R] of part `part` of `parts`, column c of Dp; the result stands in red[r * Dp + c].
template <int R> __device__ __forceinline__ void head_fold(float *red, const float (&acc)[R], int c, int part, int parts, int Dp) {
    for (int p = 0; p < parts; ++p) {  // parts one after the other, in a fixed order
        if (part == p) {
#pragma unroll
            for (int r = 0; r < R; ++r) red[r * Dp + c] = p == 0 ? acc[r] : red[r * Dp + c] + acc[r];
        }
        __syncthreads();
    }
}

template <typename T>
__global__ void __launch_bounds__(kHeadThreads) ce_head_bwd_kernel(const __grid_constant__ CeHeadArgs g, int row_ctas) {
    extern __shared__ float4 head_smem_raw[];
    __shared__ float s_weight[kHeadMaxB], s_lse[kHeadMaxB];
    __shared__ int s_label[kHeadMaxB];
    const int P = head_pitch(g.D);
    float *ws = reinterpret_cast<float *>(head_smem_raw), *xs = ws + g.V * P, *z = xs + kHeadRows * P, *red = z + g.V * kHeadRows;
    pdl_launch();
    pdl_wait();
    bool counted = false;
    if ((int)threadIdx.x < g.B) {
        const int y = g.labels[threadIdx.x];
        counted = y >= 0 && y < g.V;
        s_label[threadIdx.x] = y;
        s_lse[threadIdx.x] = g.lse[threadIdx.x];
        s_weight[threadIdx.x] = counted ? (g.drow ? g.drow[threadIdx.x] : 1.f) : 0.f;
    }
    const int n_counted = __syncthreads_count(counted);
    const float scale = g.drow ? 1.f : (g.dloss ? *g.dloss : 1.f) / (float)max(n_counted, 1);
    // threads of a column: Dp columns (a power of two), the rest of the block splits what is summed over
    int Dp = 32;
    while (Dp < g.D && Dp < kHeadThreads) Dp *= 2;
    const int parts = kHeadThreads / Dp, part = threadIdx.x / Dp;
    if ((int)blockIdx.x < row_ctas) {
        if (!g.dx) return;
        const int r0 = blockIdx.x * kHeadRows;
        head_fill(ws, (const T *)g.W, 0, g.V, g.V, g.D, P, nullptr);
        head_fill(xs, (const T *)g.x, r0, kHeadRows, g.B, g.D, P, nullptr);
        __syncthreads();
        head_logits<T>(g, ws, xs, z, P);
        __syncthreads();
        for (int i = threadIdx.x; i < g.V * kHeadRows; i += kHeadThreads) {
            const int v = i / kHeadRows, row = r0 + (i & (kHeadRows - 1));
            const float w = row < g.B ? s_weight[row] : 0.f;
            z[i] = w != 0.f ? (expf(z[i] - s_lse[row]) - (s_label[row] == v ? 1.f : 0.f)) * w : 0.f;
        }
        __syncthreads();
        for (int c0 = 0; c0 < g.D; c0 += Dp) {
            const int c = c0 + (int)(threadIdx.x & (Dp - 1));
            float acc[kHeadRows];
#pragma unroll
            for (int r = 0; r < kHeadRows; ++r) acc[r] = 0.f;
            if (c < g.D) {
#pragma unroll 4
                for (int v = part; v < g.V; v += parts) {
                    const float w = ws[v * P + c];
                    const float4 a = *reinterpret_cast<const float4 *>(z + v * kHeadRows), b = *reinterpret_cast<const float4 *>(z + v * kHeadRows + 4);
                    acc[0] = fmaf(a.x, w, acc[0]); acc[1] = fmaf(a.y, w, acc[1]); acc[2] = fmaf(a.z, w, acc[2]); acc[3] = fmaf(a.w, w, acc[3]);
                    acc[4] = fmaf(b.x, w, acc[4]); acc[5] = fmaf(b.y, w, acc[5]); acc[6] = fmaf(b.z, w, acc[6]); acc[7] = fmaf(b.w, w, acc[7]);
                }
            }
            head_fold(red, acc, c - c0, part, parts, Dp);
            for (int i = threadIdx.x; i < kHeadRows * Dp; i += kHeadThreads) {
                const int row = r0 + i / Dp, col = c0 + (i & (Dp - 1));
                // a row that does not count is zero even where W is not finite
                if (row < g.B && col < g.D) ((T *)g.dx)[(size_t)row * g.D + col] = from_f<T>(s_weight[row] != 0.f ? red[i] * scale : 0.f);
            }
            __syncthreads();
        }
    } else {
        const int v0 = ((int)blockIdx.x - row_ctas) * kHeadRows;
        const int chunk = head_chunk(g.B, g.D);
        float *xs = ws + kHeadRows * P, *dz = xs + chunk * P, *red = dz + chunk * kHeadRows;  // dz [chunk][8]
        head_fill(ws, (const T *)g.W, v0, kHeadRows, g.V, g.D, P, nullptr);
        const int s = threadIdx.x & (kHeadRows - 1), n = threadIdx.x / kHeadRows;  // an entry of the slice, and every 32nd row
        const float bias = g.bias && v0 + s < g.V ? to_f(((const T *)g.bias)[v0 + s]) : 0.f;
        float acc[kHeadMaxD / kHeadThreads][kHeadRows], db = 0.f;
#pragma unroll
        for (int q = 0; q < kHeadMaxD / kHeadThreads; ++q)
#pragma unroll
            for (int r = 0; r < kHeadRows; ++r) acc[q][r] = 0.f;
        const int col = (int)(threadIdx.x & (Dp - 1));
        for (int r0 = 0; r0 < g.B; r0 += chunk) {
            const int rows = min(chunk, g.B - r0);
            __syncthreads();  // the chunk before is read
            // a row that does not count is left out, whatever stands in it
            head_fill(xs, (const T *)g.x, r0, rows, g.B, g.D, P, s_weight + r0);
            __syncthreads();
            for (int i = n; i < rows; i += kHeadThreads / kHeadRows) {
                float d[1] = {0.f};
                const float w = s_weight[r0 + i];
                head_dots<1>(ws + s * P, xs + i * P, P, g.D, d);
                dz[i * kHeadRows + s] = w != 0.f && v0 + s < g.V ? (expf(d[0] + bias - s_lse[r0 + i]) - (s_label[r0 + i] == v0 + s ? 1.f : 0.f)) * w : 0.f;
            }
            __syncthreads();
            {   // a warp per entry
                float t = 0.f;
                for (int i = threadIdx.x & 31; i < rows; i += 32) t += dz[i * kHeadRows + (threadIdx.x >> 5)];
                db += warp_sum(t);
            }
#pragma unroll
            for (int q = 0; q < kHeadMaxD / kHeadThreads; ++q) {
                const int c = q * Dp + col;
                if (c < g.D) {
#pragma unroll 4
                    for (int i = part; i < rows; i += parts) {
                        const float xv = xs[i * P + c];
                        const float4 a = *reinterpret_cast<const float4 *>(dz + i * kHeadRows), b = *reinterpret_cast<const float4 *>(dz + i * kHeadRows + 4);
                        acc[q][0] = fmaf(a.x, xv, acc[q][0]); acc[q][1] = fmaf(a.y, xv, acc[q][1]); acc[q][2] = fmaf(a.z, xv, acc[q][2]); acc[q][3] = fmaf(a.w, xv, acc[q][3]);
                        acc[q][4] = fmaf(b.x, xv, acc[q][4]); acc[q][5] = fmaf(b.y, xv, acc[q][5]); acc[q][6] = fmaf(b.z, xv, acc[q][6]); acc[q][7] = fmaf(b.w, xv, acc[q][7]);
                    }
                }
            }
        }
        if (g.db && (threadIdx.x & 31) == 0 && v0 + (int)(threadIdx.x >> 5) < g.V) g.db[v0 + (threadIdx.x >> 5)] = db * scale;
        if (!g.dW) return;
        __syncthreads();
#pragma unroll
        for (int q = 0; q < kHeadMaxD / kHeadThreads; ++q) {
            if (q * Dp >= g.D) break;
            head_fold(red, acc[q], col, part, parts, Dp);
            for (int i = threadIdx.x; i < kHeadRows * Dp; i += kHeadThreads) {
                const int v = v0 + i / Dp, c = q * Dp + (i & (Dp - 1));
                if (v < g.V && c < g.D) {
                    const float w = red[i] * scale;
                    if (g.dw_f32) ((float *)g.dW)[(size_t)v * g.D + c] = w; else ((T *)g.dW)[(size_t)v * g.D + c] = from_f<T>(w);
                }
            }
            __syncthreads();
        }
    }
}

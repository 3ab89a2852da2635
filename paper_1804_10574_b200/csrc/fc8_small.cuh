// The gradients of small layers in one launch on the CUDA cores, part of fc8.cu: what such a call costs is its launches.
// A block has a 32 x 32 tile of dx or of dW, or 64 columns of db; the codes become the values that they stand for on their way
// into shared memory.  All of 128 K values are loaded at once: one wait for memory (with 32 at a time a layer of 128 x 128 x 128
// took 9.9 us).
constexpr int kSmallM = 32, kSmallN = 32, kSmallK = 128;

struct SmallArgs {
    const void *dy;
    const int8_t *xq, *wq;
    const float *xs, *ws;
    void *dx, *dW;
    float *db;
    int B, in, out, pitch;
    int dx_tiles, dw_tiles;
};

// C[M][N] = sum_k A(m, k) value(q[k][n]), K <= kSmallK: A is dy, K-major for dx, M-major (transposed) for dW
template <typename T, typename TC, bool A_MN>
__device__ __forceinline__ void small_tile(float (&sa)[kSmallK][kSmallM + 1], float (&sb)[kSmallK][kSmallN], const T *a, int lda, const int8_t *q, const float *scale, int pitch, TC *c, int M, int N, int K, int tile) {
    constexpr int kLoads = kSmallK * kSmallM / 256;
    const int tiles_n = (N + kSmallN - 1) / kSmallN, m0 = tile / tiles_n * kSmallM, n0 = (tile % tiles_n) * kSmallN, t = threadIdx.x;
    const int ty = t >> 4, tx = t & 15;  // rows ty and ty + 16, columns 2 tx and 2 tx + 1
    float acc[2][2] = {};
    float ra[kLoads], rs[kLoads];
    int rb[kLoads];
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {  // neighbouring lanes along the axis that lies in memory
        const int e = t + 256 * i, k = A_MN ? e / kSmallM : e % kSmallK, m = m0 + (A_MN ? e % kSmallM : e / kSmallK);
        ra[i] = k < K && m < M ? to_f(A_MN ? a[(size_t)k * lda + m] : a[(size_t)m * lda + k]) : 0.f;
        const int kb = e / kSmallN, n = n0 + e % kSmallN;
        rb[i] = kb < K && n < N ? q[(size_t)kb * pitch + n] : 0;
        rs[i] = kb < K && n < N ? scale[kb] : 0.f;
    }
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
        const int e = t + 256 * i;
        sa[A_MN ? e / kSmallM : e % kSmallK][A_MN ? e % kSmallM : e / kSmallK] = ra[i];
        sb[e / kSmallN][e % kSmallN] = act8_value<T>(rb[i], rs[i]);
    }
    __syncthreads();
#pragma unroll 16
    for (int k = 0; k < K; ++k) {
        const float2 b = *reinterpret_cast<const float2 *>(&sb[k][2 * tx]);
        const float a0 = sa[k][ty], a1 = sa[k][ty + 16];
        acc[0][0] = fmaf(a0, b.x, acc[0][0]); acc[0][1] = fmaf(a0, b.y, acc[0][1]);
        acc[1][0] = fmaf(a1, b.x, acc[1][0]); acc[1][1] = fmaf(a1, b.y, acc[1][1]);
    }
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const int m = m0 + ty + 16 * i, n = n0 + 2 * tx + j;
            if (m < M && n < N) c[(size_t)m * N + n] = from_f<TC>(acc[i][j]);
        }
}

template <typename T, typename TW> __global__ void __launch_bounds__(256) fc8_small_bwd_kernel(const __grid_constant__ SmallArgs g) {
    __shared__ __align__(8) float sa[kSmallK][kSmallM + 1], sb[kSmallK][kSmallN];
    pdl_launch();
    pdl_wait();
    int block = blockIdx.x;
    if (block < g.dx_tiles) {
        small_tile<T, T, false>(sa, sb, (const T *)g.dy, g.out, g.wq, g.ws, g.pitch, (T *)g.dx, g.B, g.in, g.out, block);
        return;
    }
    block -= g.dx_tiles;
    if (block < g.dw_tiles) {
        small_tile<T, TW, true>(sa, sb, (const T *)g.dy, g.out, g.xq, g.xs, g.pitch, (TW *)g.dW, g.out, g.in, g.B, block);
        return;
    }
    block -= g.dw_tiles;
    __shared__ float fold[4][64];
    const int l = threadIdx.x & 63, r = threadIdx.x >> 6, c = block * 64 + l;
    float a = 0.f;
    if (c < g.out) {
#pragma unroll 8
        for (int row = r; row < g.B; row += 4) a += to_f(((const T *)g.dy)[(size_t)row * g.out + c]);
    }
    fold[r][l] = a;
    __syncthreads();
    if (r == 0 && c < g.out) g.db[c] = ((fold[0][l] + fold[1][l]) + fold[2][l]) + fold[3][l];
}

// Fully connected layer on rows of 8-bit codes (act8.cuh): y = (xq xs)(wq ws)^T + bias from 32-bit integer sums, and the
// gradients of the layer from the codes that were kept, dx = dy w^, dW = dy^T x^, db = sum dy, with w^ and x^ what the codes
// stand for in the element type.
#include <algorithm>

#include "act8.cuh"
#include "common.cuh"
#include "lm_ops.h"

namespace ddg {

namespace {

constexpr int kT = 64;

template <typename T, typename TY>
__global__ void __launch_bounds__(256) fc8_fwd_kernel(const int8_t *__restrict__ xq, const float *__restrict__ xs, const int8_t *__restrict__ wq, const float *__restrict__ ws,
                                                      const T *__restrict__ bias, TY *__restrict__ y, int B, int in, int out, int pitch) {
    __shared__ int sx[kT][17], sw[kT][17];
    pdl_launch();
    pdl_wait();
    const int m0 = blockIdx.y * kT, n0 = blockIdx.x * kT, tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
    int acc[4][4] = {};
    for (int k0 = 0; k0 < in; k0 += 64) {
        __syncthreads();
        for (int i = threadIdx.x; i < kT * 16; i += 256) {
            const int r = i >> 4, c = i & 15, k = k0 + 4 * c;
            auto word = [&](const int8_t *p, int row, int rows) {
                if (row >= rows || k >= in) return 0;
                const uint32_t w = *reinterpret_cast<const uint32_t *>(p + (size_t)row * pitch + k);
                return (int)(in - k >= 4 ? w : w & ((1u << (8 * (in - k))) - 1u));  // what stands behind a row's codes is not read
            };
            sx[r][c] = word(xq, m0 + r, B);
            sw[r][c] = word(wq, n0 + r, out);
        }
        __syncthreads();
#pragma unroll
        for (int c = 0; c < 16; ++c)
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j) acc[i][j] = __dp4a(sx[ty + 16 * i][c], sw[tx + 16 * j][c], acc[i][j]);
    }
    for (int i = 0; i < 4; ++i)
        for (int j = 0; j < 4; ++j) {
            const int m = m0 + ty + 16 * i, n = n0 + tx + 16 * j;
            if (m < B && n < out) y[(size_t)m * out + n] = from_f<TY>((float)acc[i][j] * xs[m] * ws[n] + (bias ? to_f(bias[n]) : 0.f));
        }
}

// C[M][N] = sum_k A(m, k) value(B[k][n]): A is dy (K-major for dx, M-major for dW), B rows of codes with a scale each.
template <typename T, typename TC, bool A_MN>
__global__ void __launch_bounds__(256) fc8_grad_kernel(const T *__restrict__ a, const int8_t *__restrict__ q, const float *__restrict__ scale, TC *__restrict__ c, int M, int N, int K,
                                                       int lda, int pitch) {
    __shared__ float sa[16][kT + 1], sb[16][kT + 1];
    pdl_launch();
    pdl_wait();
    const int m0 = blockIdx.y * kT, n0 = blockIdx.x * kT, tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
    float acc[4][4] = {};
    for (int k0 = 0; k0 < K; k0 += 16) {
        __syncthreads();
        for (int i = threadIdx.x; i < 16 * kT; i += 256) {
            const int k = A_MN ? i / kT : i % 16, m = A_MN ? i % kT : i / 16;
            sa[k][m] = k0 + k < K && m0 + m < M ? to_f(A_MN ? a[(size_t)(k0 + k) * lda + m0 + m] : a[(size_t)(m0 + m) * lda + k0 + k]) : 0.f;
            const int kb = i / kT, n = i % kT;
            sb[kb][n] = k0 + kb < K && n0 + n < N ? act8_value<T>(q[(size_t)(k0 + kb) * pitch + n0 + n], scale[k0 + kb]) : 0.f;
        }
        __syncthreads();
#pragma unroll
        for (int k = 0; k < 16; ++k)
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j) acc[i][j] = fmaf(sa[k][ty + 16 * i], sb[k][tx + 16 * j], acc[i][j]);
    }
    for (int i = 0; i < 4; ++i)
        for (int j = 0; j < 4; ++j) {
            const int m = m0 + ty + 16 * i, n = n0 + tx + 16 * j;
            if (m < M && n < N) c[(size_t)m * N + n] = from_f<TC>(acc[i][j]);
        }
}

template <typename T> __global__ void __launch_bounds__(256) fc8_db_kernel(const T *__restrict__ dy, float *__restrict__ db, int B, int out) {
    __shared__ float fold[8][32];
    pdl_launch();
    pdl_wait();
    const int lane = threadIdx.x & 31, w = threadIdx.x >> 5, c = blockIdx.x * 32 + lane;
    float a = 0.f;
    if (c < out)
        for (int r = w; r < B; r += 8) a += to_f(dy[(size_t)r * out + c]);
    fold[w][lane] = a;
    __syncthreads();
    if (w == 0 && c < out) {
        for (int i = 1; i < 8; ++i) a += fold[i][lane];
        db[c] = a;
    }
}

template <typename T, typename TW>
int bwd_as(const void *dy, const void *xq, const float *xs, const void *wq, const float *ws, void *dx, void *dW, float *db, int B, int in, int out, const Launch &s) {
    const int pitch = act8_pitch(in);
    int n = 0;
    if (dx) {
        launch_k(fc8_grad_kernel<T, T, false>, dim3((in + kT - 1) / kT, (B + kT - 1) / kT), 256, 0, s, (const T *)dy, (const int8_t *)wq, ws, (T *)dx, B, in, out, out, pitch);
        ++n;
    }
    if (dW) {
        launch_k(fc8_grad_kernel<T, TW, true>, dim3((in + kT - 1) / kT, (out + kT - 1) / kT), 256, 0, s, (const T *)dy, (const int8_t *)xq, xs, (TW *)dW, out, in, B, out, pitch);
        ++n;
    }
    if (db) {
        launch_k(fc8_db_kernel<T>, (out + 31) / 32, 256, 0, s, (const T *)dy, db, B, out);
        ++n;
    }
    return n;
}

}  // namespace

int launch_fc8_fwd(int prec, const void *xq, const float *xs, const void *wq, const float *ws, const void *bias, void *y, int B, int in, int out, int y_f32, Launch s) {
    const dim3 grid((out + kT - 1) / kT, (B + kT - 1) / kT);
    const int pitch = act8_pitch(in);
    if (prec == P_F32) launch_k(fc8_fwd_kernel<float, float>, grid, 256, 0, s, (const int8_t *)xq, xs, (const int8_t *)wq, ws, (const float *)bias, (float *)y, B, in, out, pitch);
    else if (y_f32) launch_k(fc8_fwd_kernel<bf16, float>, grid, 256, 0, s, (const int8_t *)xq, xs, (const int8_t *)wq, ws, (const bf16 *)bias, (float *)y, B, in, out, pitch);
    else launch_k(fc8_fwd_kernel<bf16, bf16>, grid, 256, 0, s, (const int8_t *)xq, xs, (const int8_t *)wq, ws, (const bf16 *)bias, (bf16 *)y, B, in, out, pitch);
    return 1;
}

size_t fc8_workspace_bytes(int, int, int, int) { return 256; }

int launch_fc8_bwd(int prec, const void *dy, const void *xq, const float *xs, const void *wq, const float *ws, void *dx, void *dW, float *db, void *, int B, int in, int out,
                   int dw_f32, Launch s) {
    if (prec == P_F32) return bwd_as<float, float>(dy, xq, xs, wq, ws, dx, dW, db, B, in, out, s);
    return dw_f32 ? bwd_as<bf16, float>(dy, xq, xs, wq, ws, dx, dW, db, B, in, out, s) : bwd_as<bf16, bf16>(dy, xq, xs, wq, ws, dx, dW, db, B, in, out, s);
}

}  // namespace ddg

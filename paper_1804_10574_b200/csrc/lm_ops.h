// Launchers of the operators of a language-model step: dropout, RMS norm, vocabulary projection with softmax cross entropy;
// the norms around a block, rows of 8-bit codes and the linear layer on them.  As in kernels.h every launcher only enqueues on the given stream; it returns the number of launches it
// issued, or a negative value when it refused.
#pragma once
#include <cuda_runtime.h>
#include <stddef.h>

#include "kernels.h"

namespace ddg {

// ---- vocabulary projection + softmax cross entropy (linear_ce.cu) ----------------------------------------------------
// Bytes of device workspace of one call; 0 when the sizes are not supported.
size_t linear_ce_workspace_bytes(int prec, int B, int in, int out, int backward);
int launch_linear_ce_fwd(int prec, const void *x, const void *W, const void *bias, const int *labels, float *loss,
                         float *row_loss, float *lse, void *ws, int B, int in, int out, Launch s);
int launch_linear_ce_bwd(int prec, const void *x, const void *W, const void *bias, const int *labels, const float *lse,
                         const float *dloss, const float *drow, void *dx, void *dW, float *db, void *ws, int B, int in,
                         int out, int dw_f32, Launch s);
// Polls before a device-side wait of the calls of this thread gives up; negative: the default.
void linear_ce_wait_polls(int polls);
// x and W are read in place (and have to start on 16-byte boundaries) when this is true, else through a copy
bool linear_ce_in_place(int prec, int in);

// ---- RMS norm with the residual's addition (rmsnorm.cu) --------------------------------------------------------------
constexpr int kRmsMaxC = 16384, kRmsMaxRows = 1 << 30;  // row indices step by up to a few thousand in 32 bits
size_t rmsnorm_scratch_elems(int rows, int C);
// group 128 needs C % 128 == 0 and every tensor on a 16-byte boundary (y8: 8), else the launch is refused
int launch_add_rmsnorm_fwd(int prec, const void *x, const void *res, const void *gamma, void *h, void *y, void *y8,
                           float *scale8, float *rstd, int rows, int C, int group, float eps, Launch s);
int launch_add_rmsnorm_bwd(int prec, const void *dy, const void *dh, const void *h, const void *gamma, const float *rstd,
                           void *dx, float *dgamma, float *scratch, int rows, int C, Launch s);

// ---- dropout (dropout.cu) --------------------------------------------------------------------------------------------
// res nullable; threshold = drop probability in units of 2^-16
int launch_dropout(int prec, const void *x, const void *res, void *y, const unsigned long long *rng, size_t n,
                   unsigned threshold, unsigned layer, Launch s);

// ---- rows of 8-bit codes (act8.cu) -----------------------------------------------------------------------------------
// bytes from a row of codes to the next: rows that TMA can read
inline int act8_pitch(int C) { return (C + 15) / 16 * 16; }
constexpr int kAct8MaxC = 1 << 17;  // products of so many codes sum up to less than 2^31
int launch_act8_pack(int prec, const void *x, void *q, float *scale, int rows, int C, Launch s);
int launch_act8_unpack(int prec, const void *q, const float *scale, void *x, int rows, int C, Launch s);

// ---- linear layer on 8-bit codes (fc8.cu) ----------------------------------------------------------------------------
int launch_fc8_fwd(int prec, const void *xq, const float *xs, const void *wq, const float *ws, const void *bias, void *y, int B, int in, int out, int y_f32, Launch s);
size_t fc8_workspace_bytes(int prec, int B, int in, int out);
// Polls before a device-side wait of the calls of this thread gives up (these operators and the rows of codes and norms that go
// through shared memory); negative: the default.
void block8_wait_polls(int polls);
unsigned block8_polls();
int launch_fc8_bwd(int prec, const void *dy, const void *xq, const float *xs, const void *wq, const float *ws, void *dx, void *dW, float *db, void *ws_mem, int B, int in,
                   int out, int dw_f32, Launch s);

// ---- norms around a block (block_norm.cu) ----------------------------------------------------------------------------
// span: rows that share a row of the gate
int launch_block_norm_fwd(int prec, const void *b, const void *res, const void *gate, const void *post, const void *pre, void *h, void *y, void *q, float *scale,
                          float *rstd_post, float *rstd_pre, int rows, int C, int span, float alpha, float eps, Launch s);
size_t block_norm_scratch_elems(int rows, int C, int span);
int launch_block_norm_bwd(int prec, const void *dy, const void *dh, const void *b, const void *h, const void *gate, const void *post, const void *pre,
                          const float *rstd_post, const float *rstd_pre, void *db, void *dres, float *dgate, float *dpost, float *dpre, float *scratch, int rows, int C,
                          int span, float alpha, Launch s);

}  // namespace ddg

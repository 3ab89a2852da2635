// Launchers of the operators at the tail of a language-model step: dropout, RMS norm, vocabulary projection with softmax
// cross entropy.  As in kernels.h every launcher only enqueues on the given stream; it returns the number of launches it
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

}  // namespace ddg

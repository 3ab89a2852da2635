// C-ABI entry points of the operators at the tail of a language-model step (dropout, RMS norm, vocabulary projection with
// softmax cross entropy).
#include <math.h>
#include <stdio.h>

#include <initializer_list>

#include "../../include/ddg.h"
#include "common.cuh"
#include "conv_tc.h"
#include "lm_ops.h"

using namespace ddg;

namespace ddg { void set_global_error(const char *msg); }

namespace {

ddg_status refuse(ddg_status st, const char *msg) {
    set_global_error(msg);
    return st;
}
bool bad_prec(int p) { return p != DDG_FP32 && p != DDG_BF16; }
bool misaligned(const void *p, size_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) != 0; }

// Before the first launch of a call: no error of an earlier call may be pending (it would be blamed on this one), and every
// tensor has to be memory of the current device (the kernels run there).
ddg_status ready(std::initializer_list<const void *> tensors) {
    const cudaError_t e = cudaPeekAtLastError();
    if (e != cudaSuccess) {
        static thread_local char msg[256];
        snprintf(msg, sizeof(msg), "an earlier CUDA error is still pending: %s", cudaGetErrorString(e));
        return refuse(DDG_ERR_CUDA, msg);
    }
    int dev = -1;
    if (cudaGetDevice(&dev) != cudaSuccess) { cudaGetLastError(); return refuse(DDG_ERR_CUDA, "no CUDA device"); }
    for (const void *p : tensors) {
        if (!p) continue;
        cudaPointerAttributes a;
        if (cudaPointerGetAttributes(&a, p) != cudaSuccess) { cudaGetLastError(); return refuse(DDG_ERR_INVALID_ARG, "a tensor's address is not known to CUDA"); }
        if (a.type != cudaMemoryTypeDevice && a.type != cudaMemoryTypeManaged) return refuse(DDG_ERR_INVALID_ARG, "a tensor is not in device memory");
        if (a.type == cudaMemoryTypeDevice && a.device != dev) return refuse(DDG_ERR_INVALID_ARG, "a tensor is on another device than the current one");
    }
    return DDG_OK;
}
ddg_status done(int r) {
    if (r < 0) {
        const cudaError_t e = cudaGetLastError();
        return refuse(DDG_ERR_CUDA, e != cudaSuccess ? cudaGetErrorString(e) : "the kernel launcher refused the launch (tensor map or shared-memory plan)");
    }
    const cudaError_t e = cudaGetLastError();
    return e == cudaSuccess ? DDG_OK : refuse(DDG_ERR_CUDA, cudaGetErrorString(e));
}

// the sizes the tensor maps and the 32-bit indices of rows, columns and tiles can hold
bool ce_sizes_ok(int B, int in, int out) { return B >= 1 && in >= 1 && out >= 1 && B <= (1 << 24) && in <= (1 << 20) && out <= (1 << 24); }

ddg_status ce_check(int precision, const void *x, const void *W, const void *ws, size_t ws_bytes, int B, int in, int out, int backward) {
    if (linear_ce_in_place(precision, in) && (misaligned(x, 16) || misaligned(W, 16)))
        return refuse(DDG_ERR_INVALID_ARG, "linear_ce: x and W have to start on 16-byte boundaries");
    if (misaligned(ws, 256)) return refuse(DDG_ERR_INVALID_ARG, "linear_ce: the workspace has to start on a 256-byte boundary");
    if (ws_bytes < linear_ce_workspace_bytes(precision, B, in, out, backward))
        return refuse(DDG_ERR_INVALID_ARG, "linear_ce: the workspace is smaller than ddg_linear_ce_workspace_bytes says");
    return DDG_OK;
}

ddg_status dropout(int precision, const void *x, const void *res, void *y, const void *rng, size_t n, float p, unsigned layer, void *stream) {
    if (bad_prec(precision) || !x || !y || !rng) return DDG_ERR_INVALID_ARG;
    if (!(p >= 0.f && p <= 1.f)) return refuse(DDG_ERR_INVALID_ARG, "dropout: p has to be in [0, 1]");
    if (misaligned(rng, 8)) return refuse(DDG_ERR_INVALID_ARG, "dropout: rng has to start on an 8-byte boundary");
    if (n < 1) return DDG_ERR_UNSUPPORTED;
    const ddg_status st = ready({x, res, y, rng});
    if (st != DDG_OK) return st;
    return done(launch_dropout(precision, x, res, y, (const unsigned long long *)rng, n, (unsigned)rint((double)p * 65536.0), layer, (cudaStream_t)stream));
}

}  // namespace

extern "C" {

size_t ddg_linear_ce_workspace_bytes(int precision, int B, int in, int out, int backward) {
    return !bad_prec(precision) && ce_sizes_ok(B, in, out) ? linear_ce_workspace_bytes(precision, B, in, out, backward) : 0;
}

ddg_status ddg_linear_ce_fwd(int precision, const void *x, const void *W, const void *bias, const int *labels, float *loss, float *row_loss, float *lse,
                             void *workspace, size_t workspace_bytes, int B, int in, int out, void *stream) {
    if (bad_prec(precision) || !x || !W || !labels || !workspace || (!loss && !row_loss && !lse)) return DDG_ERR_INVALID_ARG;
    if (!ce_sizes_ok(B, in, out)) return DDG_ERR_UNSUPPORTED;
    ddg_status st = ce_check(precision, x, W, workspace, workspace_bytes, B, in, out, 0);
    if (st != DDG_OK) return st;
    if ((st = ready({x, W, bias, labels, loss, row_loss, lse, workspace})) != DDG_OK) return st;
    if (conv_tc_init() != 0) return DDG_ERR_CUDA;
    return done(launch_linear_ce_fwd(precision, x, W, bias, labels, loss, row_loss, lse, workspace, B, in, out, (cudaStream_t)stream));
}

ddg_status ddg_linear_ce_bwd(int precision, const void *x, const void *W, const void *bias, const int *labels, const float *lse, const float *dloss,
                             const float *drow, void *dx, void *dW, float *db, void *workspace, size_t workspace_bytes, int B, int in, int out, int dw_f32,
                             void *stream) {
    if (bad_prec(precision) || !x || !W || !labels || !lse || !workspace || (!dx && !dW && !db) || (dloss && drow)) return DDG_ERR_INVALID_ARG;
    if (dW == W) return refuse(DDG_ERR_INVALID_ARG, "linear_ce: dW may not be W");
    if (!ce_sizes_ok(B, in, out)) return DDG_ERR_UNSUPPORTED;
    ddg_status st = ce_check(precision, x, W, workspace, workspace_bytes, B, in, out, 1);
    if (st != DDG_OK) return st;
    if ((st = ready({x, W, bias, labels, lse, dloss, drow, dx, dW, db, workspace})) != DDG_OK) return st;
    if (conv_tc_init() != 0) return DDG_ERR_CUDA;
    return done(launch_linear_ce_bwd(precision, x, W, bias, labels, lse, dloss, drow, dx, dW, db, workspace, B, in, out, dw_f32, (cudaStream_t)stream));
}

void ddg_debug_linear_ce_wait_polls(int polls) { linear_ce_wait_polls(polls); }

size_t ddg_rmsnorm_scratch_elems(int rows, int C) { return rows >= 1 && rows <= kRmsMaxRows && C >= 1 && C <= kRmsMaxC ? rmsnorm_scratch_elems(rows, C) : 0; }

ddg_status ddg_add_rmsnorm_fwd(int precision, const void *x, const void *res, const void *gamma, void *h, void *y, void *y8, float *scale8, float *rstd,
                               int rows, int C, int group, float eps, void *stream) {
    if (bad_prec(precision) || !x || !gamma || (!y && !y8) || (y8 == nullptr) != (scale8 == nullptr) || (res && !h)) return DDG_ERR_INVALID_ARG;
    if (!(eps >= 0.f) || isinf(eps)) return refuse(DDG_ERR_INVALID_ARG, "add_rmsnorm: eps has to be finite and not negative");
    if (group != 0 && group != 128) return refuse(DDG_ERR_INVALID_ARG, "add_rmsnorm: group has to be 0 (a row) or 128");
    if (rows < 1 || rows > kRmsMaxRows || C < 1 || C > kRmsMaxC) return DDG_ERR_UNSUPPORTED;
    if (y8 && group != 0) {
        if (C % group != 0) return refuse(DDG_ERR_UNSUPPORTED, "add_rmsnorm: C has to be a multiple of the group");
        for (const void *p : {x, res, gamma, (const void *)h, (const void *)y, (const void *)y8})
            if (misaligned(p, 16)) return refuse(DDG_ERR_INVALID_ARG, "add_rmsnorm: with scales per group every tensor has to start on a 16-byte boundary");
    }
    const ddg_status st = ready({x, res, gamma, h, y, y8, scale8, rstd});
    if (st != DDG_OK) return st;
    return done(launch_add_rmsnorm_fwd(precision, x, res, gamma, h, y, y8, scale8, rstd, rows, C, y8 ? group : 0, eps, (cudaStream_t)stream));
}

ddg_status ddg_add_rmsnorm_bwd(int precision, const void *dy, const void *dh, const void *h, const void *gamma, const float *rstd, void *dx, float *dgamma,
                               float *scratch, int rows, int C, void *stream) {
    if (bad_prec(precision) || !dy || !h || !gamma || !rstd || !dx || !dgamma || !scratch) return DDG_ERR_INVALID_ARG;
    if (rows < 1 || rows > kRmsMaxRows || C < 1 || C > kRmsMaxC) return DDG_ERR_UNSUPPORTED;
    const ddg_status st = ready({dy, dh, h, gamma, rstd, dx, dgamma, scratch});
    if (st != DDG_OK) return st;
    return done(launch_add_rmsnorm_bwd(precision, dy, dh, h, gamma, rstd, dx, dgamma, scratch, rows, C, (cudaStream_t)stream));
}

ddg_status ddg_dropout_fwd(int precision, const void *x, const void *res, void *y, const void *rng, size_t n, float p, unsigned layer, void *stream) {
    return dropout(precision, x, res, y, rng, n, p, layer, stream);
}

ddg_status ddg_dropout_bwd(int precision, const void *dy, void *dx, const void *rng, size_t n, float p, unsigned layer, void *stream) {
    return dropout(precision, dy, nullptr, dx, rng, n, p, layer, stream);
}

}  // extern "C"

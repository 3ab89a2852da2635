"""Per-kernel sweep over the ResNet-110 layer shapes, over the tail of a language-model step (dropout, RMS norm, vocabulary
projection with cross entropy) and over a block around a linear layer in 8 bits, through the single-kernel C-ABI entry points.

    python -m paper_1804_10574_b200.kernel_sweep [--batch 1024] [--only NAME] [--iters 20] [--json] [--warm]

Times every kernel alone with CUDA events on its stream, flushing L2 between launches, and prints the algorithmic
bytes and flops per launch against the measured HBM / bf16 tensor peaks (MEASURED_PEAKS.json at the repository root,
else the fallback 6650 GB/s and 1590 TFLOP/s).  Inputs: bf16 N(0,1) activations and gradients, He-normal filters.
"""
import argparse
import json
import os

import numpy as np
import torch

from . import binding

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def peaks():
    try:
        p = json.load(open(os.path.join(ROOT, "MEASURED_PEAKS.json")))
        return p["hbm_gbs"], p["bf16_tflops"], "measured"
    except Exception:
        return 6650.0, 1590.0, "fallback"


def timed(fn, iters, flush):
    for _ in range(3):
        fn()
    ts = []
    s = torch.cuda.current_stream()
    for _ in range(iters):
        if flush is not None:
            flush.zero_()
        else:
            torch.cuda._sleep(200000)   # keeps the GPU busy without touching L2 while the host enqueues what follows
        e0, e1 = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
        e0.record(s)
        fn()
        e1.record(s)
        e1.synchronize()
        ts.append(e0.elapsed_time(e1) * 1e-3)
    ts = sorted(ts)
    if len(ts) >= 6:             # event stamps tick every ~2 us: averaging resolves below that, the median cannot
        ts = ts[1:-1]
    return float(np.mean(ts))


def cases(B):
    bf = torch.bfloat16
    out = []

    def conv(H, Ci, Co, st):
        Ho = (H - 1) // st + 1
        x = torch.randn(B, H, H, Ci, device="cuda").to(bf)
        dy = torch.randn(B, Ho, Ho, Co, device="cuda").to(bf)
        w = (torch.randn(Co, Ci, 3, 3, device="cuda") * (2.0 / (9 * Ci)) ** 0.5).to(bf)
        y, dx = torch.empty_like(dy), torch.empty_like(x)
        dw = torch.empty(Co, Ci, 3, 3, device="cuda")
        sc = torch.empty(max(1, binding.conv3x3_wgrad_scratch_elems(B, H, H, Ci, Co, st)), device="cuda")
        flops = 2.0 * 9 * Ci * Co * B * Ho * Ho
        io = (x.numel() + dy.numel()) * 2
        tag = "%d->%d %dx%d s%d" % (Ci, Co, H, H, st)
        tc = binding.tensor_core_path(B, H, H, Ci, Co, st)
        keep = (x, dy, w, y, dx, dw, sc)
        if tc & 1 and st == 1 and Ci == Co:   # as in the training step: filter image arranged beforehand (by the optimiser update)
            pk = torch.empty(binding.conv3x3_packed_bytes(B, H, H, Ci), dtype=torch.uint8, device="cuda")
            binding.conv3x3_pack(w, pk, Ci)
            out.append(("conv_fwd " + tag, lambda: binding.conv3x3_packed(0, x, w, pk, y, B, H, H, Ci), io, flops, 1, keep + (pk,)))
            out.append(("conv_dgrad " + tag, lambda: binding.conv3x3_packed(1, dy, w, pk, dx, B, H, H, Ci), io, flops, 1, keep + (pk,)))
        else:
            out.append(("conv_fwd " + tag, lambda: binding.conv3x3_fwd(1, x, w, y, B, H, H, Ci, Co, st), io, flops, tc & 1, keep))
            out.append(("conv_dgrad " + tag, lambda: binding.conv3x3_dgrad(1, dy, w, dx, B, H, H, Ci, Co, st), io, flops, tc & 1, keep))
        out.append(("conv_wgrad " + tag, lambda: binding.conv3x3_wgrad(1, x, dy, dw, sc, B, H, H, Ci, Co, st), io, flops, (tc >> 1) & 1, keep))

    for H, Ci, Co, st in ((32, 16, 16, 1), (16, 32, 32, 1), (8, 64, 64, 1), (32, 16, 32, 2), (16, 32, 64, 2), (32, 3, 16, 1)):
        conv(H, Ci, Co, st)

    def bn(H, C):
        HW = H * H
        x = torch.randn(B, HW, C, device="cuda").to(bf)
        r, dout = torch.randn_like(x), torch.randn_like(x)
        g, b = torch.ones(C, device="cuda").to(bf), torch.zeros(C, device="cuda").to(bf)
        y, dx = torch.empty_like(x), torch.empty_like(x)
        m, i, dg, db = (torch.empty(C, device="cuda") for _ in range(4))
        sc = torch.zeros(binding.bn_scratch_elems(C), device="cuda")
        keep = (x, r, dout, g, b, y, dx, m, i, dg, db, sc)
        n = x.numel() * 2
        out.append(("bn_relu_residual_fwd C%d %dx%d" % (C, H, H),
                    lambda: binding.bn_fwd(1, x, g, b, r, y, m, i, sc, B, HW, C, 1), 4 * n, 0.0, 0, keep))   # x twice, res, y
        out.append(("bn_relu_bwd C%d %dx%d" % (C, H, H),
                    lambda: binding.bn_bwd(1, dout, y, x, g, m, i, dx, dg, db, sc, B, HW, C, 1), 7 * n, 0.0, 0, keep))

    for H, C in ((32, 16), (16, 32), (8, 64)):
        bn(H, C)

    n = 1733812
    w, v, gr = (torch.randn(n, device="cuda") for _ in range(3))
    wv = torch.empty(n, dtype=bf, device="cuda")
    out.append(("sgd_update 1.73M params", lambda: binding.sgd_update(1, w, v, gr, wv, n, 0.01, 0.9, 5e-4), n * 22, 0.0, 0, (w, v, gr, wv)))
    return out + tail_cases(B) + block_cases(B)


def tail_cases(B, D=1024, V=32000):
    """The tail of a language-model step on B rows: bytes and flops that the operations cannot do without (the backward
    pass of the projection multiplies half as much again: it computes the logits a second time)."""
    bf = torch.bfloat16
    x, res, dy, dh = (torch.randn(B, D, device="cuda").to(bf) for _ in range(4))
    g = torch.ones(D, device="cuda").to(bf)
    w = (torch.randn(V, D, device="cuda") * D ** -0.5).to(bf)
    labels = torch.randint(0, V, (B,), device="cuda", dtype=torch.int32)
    rng = torch.tensor([1, 0], dtype=torch.int64, device="cuda")
    y, h, dx, dw = torch.empty_like(x), torch.empty_like(x), torch.empty_like(x), torch.empty_like(w)
    q = torch.empty(B, D, dtype=torch.uint8, device="cuda")
    loss, rstd, lse, dg, sc8 = (torch.ones(n, device="cuda") for n in (1, B, B, D, B * D // 128))
    sc = torch.empty(binding.rmsnorm_scratch_elems(B, D), device="cuda")
    ws = torch.empty(max(binding.linear_ce_workspace_bytes(1, B, D, V, k) for k in (False, True)), dtype=torch.uint8, device="cuda")
    keep = (x, res, dy, dh, g, w, labels, rng, y, h, dx, dw, q, loss, rstd, lse, dg, sc8, sc, ws)
    binding.linear_ce_fwd(1, x, w, None, labels, loss, None, lse, ws, B, D, V)
    n, flops, tag = B * D * 2, 2.0 * B * D * V, "%dx%d" % (B, D)
    wtag = tag + "x%d" % V
    return [
        ("dropout_residual_fwd " + tag, lambda: binding.dropout_fwd(1, x, res, y, rng, B * D, 0.1), 3 * n, 0.0, 0, keep),
        ("dropout_bwd " + tag, lambda: binding.dropout_bwd(1, dy, dx, rng, B * D, 0.1), 2 * n, 0.0, 0, keep),
        ("add_rmsnorm_fwd " + tag, lambda: binding.add_rmsnorm_fwd(1, x, res, g, h, y, None, None, rstd, B, D), 4 * n, 0.0, 0, keep),
        ("add_rmsnorm_fwd e4m3 " + tag, lambda: binding.add_rmsnorm_fwd(1, x, res, g, h, None, q, sc8, rstd, B, D, 128), 3 * n + n // 2, 0.0, 0, keep),
        ("add_rmsnorm_bwd " + tag, lambda: binding.add_rmsnorm_bwd(1, dy, dh, x, g, rstd, dx, dg, sc, B, D), 4 * n, 0.0, 0, keep),
        ("linear_ce_fwd " + wtag, lambda: binding.linear_ce_fwd(1, x, w, None, labels, loss, None, lse, ws, B, D, V), n + V * D * 2, flops, 1, keep),
        ("linear_ce_bwd " + wtag, lambda: binding.linear_ce_bwd(1, x, w, None, labels, lse, None, None, dx, dw, None, ws, B, D, V),
         2 * (n + V * D * 2), 2 * flops, 1, keep),
    ]


def block_cases(B, D=4096, F=4096):
    """A block around a linear layer in 8 bits, on B rows: norms with gate and residual scale, rows of codes, the layer's
    product on codes and its gradients."""
    bf = torch.bfloat16
    b, res, dy, dh = (torch.randn(B, D, device="cuda").to(bf) for _ in range(4))
    gate, post, pre = (torch.ones(1, D, device="cuda").to(bf) for _ in range(3))
    w, dz = (torch.randn(F, D, device="cuda") * D ** -0.5).to(bf), torch.randn(B, F, device="cuda").to(bf)
    h, y, db, dres, z, dw = torch.empty_like(b), torch.empty_like(b), torch.empty_like(b), torch.empty_like(b), torch.empty_like(dz), torch.empty(F, D, device="cuda")
    q, wq = (torch.empty(n, binding.act8_pitch(D), dtype=torch.int8, device="cuda") for n in (B, F))
    r1, r2, qs, ws, dg, dp1, dp2, dbias = (torch.ones(n, device="cuda") for n in (B, B, B, F, D, D, D, F))
    sc = torch.empty(binding.block_norm_scratch_elems(B, D, B), device="cuda")
    work = torch.empty(binding.fc8_workspace_bytes(1, B, D, F), dtype=torch.uint8, device="cuda")
    keep = (b, res, dy, dh, gate, post, pre, w, dz, h, y, db, dres, z, dw, q, wq, r1, r2, qs, ws, dg, dp1, dp2, dbias, sc, work)
    binding.act8_pack(1, w, wq, ws, F, D)
    binding.act8_pack(1, b, q, qs, B, D)
    n, wn, flops, tag, wtag = B * D * 2, F * D, 2.0 * B * D * F, "%dx%d" % (B, D), "%dx%dx%d" % (B, D, F)
    return [
        ("block_norm_fwd " + tag, lambda: binding.block_norm_fwd(1, b, res, gate, post, pre, h, y, None, None, r1, r2, B, D, B), 4 * n, 0.0, 0, keep),
        ("block_norm_fwd codes " + tag, lambda: binding.block_norm_fwd(1, b, res, gate, post, pre, h, None, q, qs, r1, r2, B, D, B), 3 * n + n // 2, 0.0, 0, keep),
        ("block_norm_bwd " + tag, lambda: binding.block_norm_bwd(1, dy, dh, b, h, gate, post, pre, r1, r2, db, dres, dg, dp1, dp2, sc, B, D, B), 6 * n, 0.0, 0, keep),
        ("act8_pack " + tag, lambda: binding.act8_pack(1, b, q, qs, B, D), n + n // 2, 0.0, 0, keep),
        ("act8_unpack " + tag, lambda: binding.act8_unpack(1, q, qs, y, B, D), n + n // 2, 0.0, 0, keep),
        ("fc8_fwd " + wtag, lambda: binding.fc8_fwd(1, q, qs, wq, ws, None, z, B, D, F), B * D + wn + B * F * 2, flops, 1, keep),
        ("fc8_bwd dx " + wtag, lambda: binding.fc8_bwd(1, dz, None, None, wq, ws, db, None, None, work, B, D, F), wn + B * F * 2 + n, flops, 1, keep),
        ("fc8_bwd dW " + wtag, lambda: binding.fc8_bwd(1, dz, q, qs, None, None, None, dw, None, work, B, D, F, True), B * D + B * F * 2 + 4 * wn, flops, 1, keep),
        ("fc8_bwd dx dW db " + wtag, lambda: binding.fc8_bwd(1, dz, q, qs, wq, ws, db, dw, dbias, work, B, D, F, True), B * D + wn + B * F * 2 + n + 4 * wn, 2 * flops, 1, keep),
    ]


def main():
    ap = argparse.ArgumentParser()
    ap.add_argument("--batch", type=int, default=1024)
    ap.add_argument("--only", default="")
    ap.add_argument("--iters", type=int, default=20)
    ap.add_argument("--json", action="store_true")
    ap.add_argument("--warm", action="store_true", help="do not flush L2 between launches (operands as the previous "
                    "kernel of a training step leaves them)")
    a = ap.parse_args()
    hbm, tf, src = peaks()
    flush = None if a.warm else torch.empty(256 << 20, dtype=torch.uint8, device="cuda")
    rows = []
    for name, fn, nbytes, flops, tc, _keep in cases(a.batch):
        if a.only and a.only not in name:
            continue
        dt = timed(fn, a.iters, flush)
        rows.append(dict(kernel=name, tensor_core=bool(tc), us=dt * 1e6, gbs=nbytes / dt / 1e9, hbm_frac=nbytes / dt / 1e9 / hbm,
                         tflops=flops / dt / 1e12, tensor_frac=flops / dt / 1e12 / tf))
    if a.json:
        print(json.dumps(dict(batch=a.batch, peaks=dict(hbm_gbs=hbm, bf16_tflops=tf, source=src), rows=rows)))
        return
    print("batch %d; peaks (%s): HBM %.0f GB/s, bf16 %.0f TFLOP/s" % (a.batch, src, hbm, tf))
    print("%-34s %3s %9s %9s %7s %9s %7s" % ("kernel", "tc", "us", "GB/s", "of HBM", "TFLOP/s", "of bf16"))
    for r in rows:
        print("%-34s %3s %9.1f %9.0f %6.1f%% %9.1f %6.1f%%" % (r["kernel"], "yes" if r["tensor_core"] else "no", r["us"], r["gbs"],
                                                              100 * r["hbm_frac"], r["tflops"], 100 * r["tensor_frac"]))
    if any(r["kernel"].endswith("3->16 32x32 s1") for r in rows):
        print("3->16: the single-kernel entry points take the 3-channel tensor as it is (CUDA-core kernels).  The bf16 training "
              "step never launches these: its input shim stores the image zero-padded to 16 channels and the stem runs on the "
              "16->16 tensor-core kernels above (forward and weight gradient; the input needs no gradient).")


if __name__ == "__main__":
    main()

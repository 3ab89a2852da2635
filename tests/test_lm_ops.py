"""Dropout, RMS norm with the residual's addition, and the vocabulary projection with softmax cross entropy, against
plain implementations in 64 bits.

Tolerances count roundings.  A rounding to a type is off by at most U[type] relative to the value (half a step).  The
tensor cores add 16 products and the accumulator at a time; every such step is taken to lose at most four units of 2^-24
of the sum of the absolute values (the products' alignment and the accumulator's truncation)."""
import math
import os
import subprocess
import sys

import numpy as np
import pytest
import torch

U = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}
DT = {0: torch.float32, 1: torch.bfloat16}
PREC = pytest.mark.parametrize("prec", [0, 1], ids=["fp32", "bf16"])
gpu = pytest.mark.gpu
NAN, INF = float("nan"), float("inf")


@pytest.fixture
def binding():
    from paper_1804_10574_b200 import binding as b
    return b


def randn(*size, seed, prec, std=1.0, mean=0.0):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return torch.empty(size, device="cuda", dtype=torch.float32).normal_(mean, std, generator=g).to(DT[prec])


def f32(*size, fill=7.0):
    return torch.full(size, fill, dtype=torch.float32, device="cuda")


def within(got, ref, tol, what):
    """got within tol of ref elementwise; NaN and infinities in the same places."""
    got, ref, tol = got.double(), ref.double(), torch.as_tensor(tol, dtype=torch.float64, device="cuda").expand_as(ref)
    assert torch.equal(torch.isnan(got), torch.isnan(ref)), what
    fine = torch.isfinite(ref)
    assert torch.equal(got[~fine & ~torch.isnan(ref)], ref[~fine & ~torch.isnan(ref)]), what
    over = ((got - ref).abs() - tol)[fine]
    if over.numel():
        i = int(over.argmax())
        assert float(over[i]) <= 0, "%s: off by %.3e, %.3e allowed, value %.3e" % (what, float((got - ref).abs()[fine][i]), float(tol[fine][i]), float(ref[fine][i]))


# ---- vocabulary projection with softmax cross entropy ---------------------------------------------------------------
class Ce:
    """Inputs, the 64-bit reference and its tolerances."""

    def __init__(self, B, D, V, prec, bias=False, ignored=0.0, seed=0, logit_std=2.0):
        self.B, self.D, self.V, self.prec = B, D, V, prec
        self.x = randn(B, D, seed=seed + 1, prec=prec)
        self.w = randn(V, D, seed=seed + 2, prec=prec, std=logit_std / math.sqrt(D))
        self.bias = randn(V, seed=seed + 3, prec=prec) if bias else None
        g = torch.Generator(device="cuda")
        g.manual_seed(seed + 4)
        self.labels = torch.randint(0, V, (B,), device="cuda", generator=g, dtype=torch.int32)
        if ignored:
            self.labels[torch.rand(B, device="cuda", generator=g) < ignored] = -1

    def reference(self, drow=None, dloss=1.0, dz_u=None):
        x, w = self.x.double(), self.w.double()
        counted = (self.labels >= 0) & (self.labels < self.V)
        x = torch.where(counted[:, None], x, torch.nan_to_num(x, nan=0.0, posinf=0.0, neginf=0.0))
        z = x @ w.t()
        mass = x.abs() @ w.abs().t()
        if self.bias is not None:
            z = z + self.bias.double()
            mass = mass + torch.nan_to_num(self.bias.double(), neginf=0.0).abs()
        parts = 6 if self.prec == 0 else 1
        # steps of the accumulator; the terms an fp32 product leaves out (m l, l m, l l and what l rounds off) are below
        # 4 x 2^-24; adding the bias rounds once
        ez = (4 * parts * math.ceil(self.D / 16) + 8) * 2.0 ** -24 * mass
        self.z, self.ez = z, ez
        self.lse = torch.logsumexp(z, 1)
        top = z.amax(1)
        # exp2 and its argument: 2^-22 and 2 roundings of |z - max| (terms far below the maximum weigh less than
        # 2^-24 |z - max| exp(z - max) < 2^-24); sums of V terms in pieces of 128 and a tree: 64 + 32 roundings; the
        # logarithm's and the sum's final roundings
        self.e_lse = torch.softmax(z, 1).mul(ez).sum(1) * 1.01 + 2.0 ** -21 + 100 * 2.0 ** -24 + 4 * 2.0 ** -24 * (top.abs() + self.lse.abs())
        y = self.labels.clamp(0, self.V - 1).long()[:, None]
        zl = z.gather(1, y)[:, 0]
        self.row = torch.where(counted, self.lse - zl, 0.0)
        self.e_row = self.e_lse + ez.gather(1, y)[:, 0] + 2.0 ** -23 * (self.lse.abs() + zl.abs())
        n = int(counted.sum())
        self.loss = self.row.sum() / max(1, n)
        self.e_loss = torch.where(counted, self.e_row, 0.0).sum() / max(1, n) + 2.0 ** -23 * self.loss.abs()
        g = drow.double() if drow is not None else torch.full_like(self.row, dloss / max(1, n))
        g = torch.where(counted, g, 0.0)
        p = torch.softmax(z, 1)
        hit = torch.zeros_like(p).scatter_(1, y, 1.0)
        dz = (p - hit) * g[:, None]
        dz = torch.where(counted[:, None], dz, 0.0)
        # p: the logit's and lse's errors, exp2 as above; then the subtraction's, the weight's and the scale's roundings
        ep = p * (ez + self.e_lse[:, None] + 2.0 ** -21 + 2.0 ** -23 * (z - self.lse[:, None]).abs())
        ep = torch.where(counted[:, None], (ep + 2.0 ** -24) * g.abs()[:, None], 0.0)
        # dz as the products see it: one, two or three terms of bf16
        edz = ep + dz.abs() * (2.0 ** -8 if self.prec == 1 else 2.0 ** -24)
        edz16 = ep + dz.abs() * (2.0 ** -16 if self.prec == 1 else 2.0 ** -24)
        self.db, self.e_db = dz.sum(0), ep.sum(0) * 1.01 + 64 * 2.0 ** -24 * dz.abs().sum(0)
        aw, ax, az = w.abs(), x.abs(), dz.abs()
        steps_v, steps_b = 4 * parts * math.ceil(self.V / 16) + 80, 4 * parts * math.ceil(self.B / 16) + 16
        self.dx = dz @ w
        self.e_dx = edz @ aw + steps_v * 2.0 ** -24 * (az @ aw) + U[DT[self.prec]] * self.dx.abs() + 1e-30
        self.dw = dz.t() @ x
        self.e_dw = edz.t() @ ax + steps_b * 2.0 ** -24 * (az.t() @ ax) + U[DT[self.prec]] * self.dw.abs() + 1e-30
        self.e_dw32 = edz16.t() @ ax + 2 * steps_b * 2.0 ** -24 * (az.t() @ ax) + 2.0 ** -24 * self.dw.abs() + 1e-30
        return self

    def fwd(self, b, stream=None):
        ws = torch.full((b.linear_ce_workspace_bytes(self.prec, self.B, self.D, self.V, False),), 255, dtype=torch.uint8, device="cuda")
        loss, row, lse = f32(1), f32(self.B), f32(self.B)
        b.linear_ce_fwd(self.prec, self.x, self.w, self.bias, self.labels, loss, row, lse, ws, self.B, self.D, self.V, stream)
        return loss, row, lse

    def bwd(self, b, lse, dloss=None, drow=None, want="xwb", dw_f32=False, stream=None):
        ws = torch.full((b.linear_ce_workspace_bytes(self.prec, self.B, self.D, self.V, True),), 255, dtype=torch.uint8, device="cuda")
        dx = torch.full_like(self.x, 7.0) if "x" in want else None
        dw = torch.full(self.w.shape, 7.0, dtype=torch.float32 if dw_f32 else self.w.dtype, device="cuda") if "w" in want else None
        db = f32(self.V) if "b" in want else None
        b.linear_ce_bwd(self.prec, self.x, self.w, self.bias, self.labels, lse, dloss, drow, dx, dw, db, ws, self.B, self.D, self.V, dw_f32, stream)
        return dx, dw, db


CE_SHAPES = [(1, 8, 1), (1, 64, 100), (3, 5, 7), (128, 64, 100), (130, 72, 257), (257, 264, 513), (300, 521, 1000), (33, 1000, 4099),
             (2, 4096, 300), (511, 16, 255), (64, 2048, 12000),
             (16, 256, 20000), (20, 136, 3001), (65, 128, 640), (2050, 136, 520),
             (256, 64, 100), (200, 63, 90), (40, 512, 50), (9, 300, 60),
             (11, 89, 5000), (4, 1021, 1500), (16, 3100, 600), (16, 3300, 500), (7, 132, 1)]


@gpu
@PREC
@pytest.mark.parametrize("shape", CE_SHAPES, ids=lambda s: "x".join(map(str, s)))
def test_linear_ce_forward(binding, shape, prec):
    """One row to several tiles; widths and vocabularies that fill no tile, widths that TMA cannot read in place."""
    for bias, ignored in ((False, 0.0), (True, 0.3)):
        c = Ce(*shape, prec, bias, ignored, seed=5).reference()
        loss, row, lse = c.fwd(binding)
        within(lse, c.lse, c.e_lse, "lse")
        within(row, c.row, c.e_row, "row_loss")
        within(loss[0], c.loss, c.e_loss, "loss")


@gpu
@PREC
@pytest.mark.parametrize("shape", CE_SHAPES, ids=lambda s: "x".join(map(str, s)))
def test_linear_ce_backward(binding, shape, prec):
    for bias, ignored, dw_f32 in ((False, 0.0, False), (True, 0.3, True)):
        c = Ce(*shape, prec, bias, ignored, seed=6).reference(dloss=0.75)
        dx, dw, db = c.bwd(binding, c.lse.float(), dloss=f32(1, fill=0.75), dw_f32=dw_f32)
        within(dx, c.dx, c.e_dx, "dx")
        within(dw, c.dw, c.e_dw32 if dw_f32 else c.e_dw, "dW")
        within(db, c.db, c.e_db, "db")


# one of each way a call is worked: a small head, at most 64 rows, more rows
WAYS = pytest.mark.parametrize("shape", [(140, 64, 300), (45, 136, 3000), (300, 136, 777), (14, 200, 2000)], ids=["head", "few_rows", "rows", "fewest_rows"])


@gpu
@PREC
@WAYS
def test_linear_ce_row_gradients(binding, shape, prec):
    """drow: a gradient of its own for every row, zeros and signs among them; each output asked for alone."""
    c = Ce(*shape, prec, True, 0.2, seed=7)
    drow = torch.linspace(-2, 2, c.B, device="cuda")
    drow[5] = 0.0
    c.reference(drow=drow)
    lse = c.lse.float()
    full = c.bwd(binding, lse, drow=drow)
    for got, ref, tol, what in zip(full, (c.dx, c.dw, c.db), (c.e_dx, c.e_dw, c.e_db), ("dx", "dW", "db")):
        within(got, ref, tol, what)
    for k, want in enumerate("xwb"):
        assert torch.equal(c.bwd(binding, lse, drow=drow, want=want)[k], full[k]), want


@gpu
@pytest.mark.parametrize("prec,D,V", [(1, 40, 17000), (0, 40, 6000), (1, 600, 17000), (1, 601, 17000)])
def test_linear_ce_backward_in_chunks(binding, prec, D, V):
    """More rows times vocabulary than one chunk of dz holds: sums over chunks, a short last one; with splits, and with
    tiles enough without."""
    c = Ce(8200, D, V, prec, True, 0.1, seed=8)
    lse = c.fwd(binding)[2]
    dx, dw, db = c.bwd(binding, lse)
    c.reference()
    within(lse, c.lse, c.e_lse, "lse")
    within(dx, c.dx, c.e_dx, "dx")
    within(dw, c.dw, c.e_dw, "dW")
    within(db, c.db, c.e_db, "db")


@gpu
@PREC
@WAYS
def test_linear_ce_rows_that_do_not_count(binding, shape, prec):
    """Labels outside the vocabulary leave a row out, whatever stands in it; without any row the results are zero."""
    c = Ce(*shape, prec, True, seed=9)
    c.labels[3], c.labels[7], c.labels[c.B - 1], c.labels[10] = -1, c.V, -2 ** 31, 2 ** 31 - 1
    c.x[3], c.x[7, 5], c.x[c.B - 1, 0], c.x[10] = NAN, INF, -INF, torch.finfo(c.x.dtype).min
    c.reference()
    loss, row, lse = c.fwd(binding)
    counted = (c.labels >= 0) & (c.labels < c.V)
    within(row, c.row, torch.where(counted, c.e_row, 0.0), "row_loss")
    within(loss[0], c.loss, c.e_loss, "loss")
    within(lse[counted], c.lse[counted], c.e_lse[counted], "lse")
    dx, dw, db = c.bwd(binding, lse)
    within(dx, c.dx, torch.where(counted[:, None], c.e_dx, 0.0), "dx")
    within(dw, c.dw, c.e_dw, "dW")
    within(db, c.db, c.e_db, "db")
    c.labels.fill_(-1)
    loss, row, lse = c.fwd(binding)
    assert float(loss[0]) == 0.0 and not row.any()
    for g in c.bwd(binding, lse):
        assert not g.any()


@gpu
@PREC
@pytest.mark.parametrize("rows,width", [(40, 32), (40, 64), (300, 64), (12, 64)], ids=["head", "few_rows", "rows", "fewest_rows"])
def test_linear_ce_masked_vocabulary(binding, rows, width, prec):
    """A bias of minus infinity or of the type's lowest value takes entries out of the softmax, whole tiles of them too; a
    label among them has infinite loss."""
    c = Ce(rows, width, 900, prec, True, seed=10)
    c.bias[0:600] = -INF
    c.bias[700:710] = torch.finfo(c.bias.dtype).min
    c.labels.clamp_(min=710)
    c.labels[4] = 5
    loss, row, lse = c.fwd(binding)
    z = c.x.double() @ c.w.double().t() + c.bias.double()
    ref = torch.logsumexp(z, 1)
    tol = (8 * 6 * 4 + 300) * 2.0 ** -24 * 64
    within(lse, ref, tol, "lse")
    assert math.isinf(float(row[4])) and math.isinf(float(loss[0]))
    keep = torch.arange(rows, device="cuda") != 4
    within(row[keep], (ref - z.gather(1, c.labels.long()[:, None])[:, 0])[keep], tol, "row_loss")
    c.labels[4] = 800
    lse = c.fwd(binding)[2]
    dx, dw, db = c.bwd(binding, lse)
    assert not dw[0:600].any() and not dw[700:710].any() and not db[0:600].any()
    assert torch.isfinite(dx).all() and torch.isfinite(dw).all() and torch.isfinite(db).all()


@gpu
@PREC
def test_linear_ce_non_finite_rows_stay_their_own(binding, prec):
    """NaN in a row that counts: its own loss and dx are NaN, the other rows' are not touched."""
    c = Ce(300, 64, 600, prec, False, seed=11)
    clean_loss, clean_row, clean_lse = c.fwd(binding)
    clean_dx = c.bwd(binding, clean_lse)[0]
    c.x[200, 3] = NAN
    loss, row, lse = c.fwd(binding)
    assert math.isnan(float(loss[0])) and math.isnan(float(row[200])) and math.isnan(float(lse[200]))
    keep = torch.arange(300, device="cuda") != 200
    assert torch.equal(row[keep], clean_row[keep]) and torch.equal(lse[keep], clean_lse[keep])
    dx = c.bwd(binding, lse)[0]
    assert torch.isnan(dx[200]).all() and torch.equal(dx[keep], clean_dx[keep])


@gpu
@PREC
def test_linear_ce_large_logits(binding, prec):
    """Logits of hundreds: the maximum is subtracted before the exponential; p is zero or one for most."""
    c = Ce(70, 128, 1500, prec, False, seed=12, logit_std=120.0).reference()
    loss, row, lse = c.fwd(binding)
    within(lse, c.lse, c.e_lse, "lse")
    within(row, c.row, c.e_row, "row_loss")
    assert float(lse.max()) > 200
    dx, dw, _ = c.bwd(binding, lse)
    within(dx, c.dx, c.e_dx, "dx")
    within(dw, c.dw, c.e_dw, "dW")


@gpu
def test_linear_ce_gradient_against_differences(binding):
    """The loss's change along a direction of x, of W and of the bias, by central differences of the forward pass."""
    c = Ce(96, 80, 500, 0, True, 0.2, seed=13)
    dx, dw, db = c.bwd(binding, c.fwd(binding)[2])
    h = 2.0 ** -5
    for name, grad in (("x", dx), ("w", dw), ("bias", db)):
        t = getattr(c, name)
        d = randn(*t.shape, seed=14, prec=0)
        d /= d.norm()
        kept, at = t.clone(), []
        for s in (h, -h):
            t.copy_(kept + s * d)
            at.append(float(c.fwd(binding)[0]))
        t.copy_(kept)
        slope, want = (at[0] - at[1]) / (2 * h), float((grad.double() * d.double()).sum())
        # the loss is rounded to 2^-24 of ~8 and summed from rows within 1e-6: 2 x 2e-6 / 2h; the third derivative of the
        # loss along a unit direction is below the logits' change cubed, at most max |W row|^3 < 27 for x and |x row|^3 /
        # ... for W a single entry of the direction is below 1/10 of it: h^2 / 6 x 27 / 96 bounds both
        assert abs(slope - want) < 2e-6 / h + h * h / 6 * 27 / 96, (name, slope, want)


@gpu
@PREC
def test_linear_ce_other_stream_and_recorded(binding, prec):
    """On a stream of its own; forward and backward recorded into a graph and replayed on new inputs in the same
    buffers; the same bits every time."""
    c = Ce(300, 72, 900, prec, True, 0.2, seed=15)
    other = Ce(300, 72, 900, prec, True, 0.5, seed=16)
    ref = [c.fwd(binding), other.fwd(binding)]
    refs = [r + c_.bwd(binding, r[2]) for c_, r in zip((c, other), ref)]
    stream = torch.cuda.Stream()
    n, d, v = 300, 72, 900
    ws = torch.empty(max(binding.linear_ce_workspace_bytes(prec, n, d, v, k) for k in (False, True)), dtype=torch.uint8, device="cuda")
    out = [f32(1), f32(n), f32(n), torch.empty_like(c.x), torch.empty_like(c.w), f32(v)]
    torch.cuda.synchronize()

    def step():
        s = stream.cuda_stream
        binding.linear_ce_fwd(prec, c.x, c.w, c.bias, c.labels, out[0], out[1], out[2], ws, n, d, v, s)
        binding.linear_ce_bwd(prec, c.x, c.w, c.bias, c.labels, out[2], None, None, out[3], out[4], out[5], ws, n, d, v, False, s)

    step()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(out, refs[0]))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        step()
    for k, src in enumerate((c, other, c)):
        if k:
            kept = [t.clone() for t in (src.x, src.w, src.bias, src.labels)] if src is other else first
            for dst, t in zip((c.x, c.w, c.bias, c.labels), kept):
                dst.copy_(t)
        else:
            first = [t.clone() for t in (c.x, c.w, c.bias, c.labels)]
        for o in out:
            o.fill_(3.0)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, refs[k % 2])), k


@gpu
@PREC
@pytest.mark.parametrize("shape", [(128, 64, 100), (200, 63, 90), (40, 512, 50), (20, 136, 3001), (300, 72, 900)], ids=lambda s: "x".join(map(str, s)))
def test_linear_ce_gradient_over_the_rows(binding, shape, prec):
    """dx may be x itself: the same bits as into a buffer of its own where both take the same kernels, within the
    tolerance everywhere."""
    c = Ce(*shape, prec, True, 0.2, seed=19).reference()
    x, lse = c.x.clone(), c.lse.float()
    ws = torch.empty(binding.linear_ce_workspace_bytes(prec, *shape, True), dtype=torch.uint8, device="cuda")
    dw, db = torch.empty_like(c.w), f32(c.V)
    binding.linear_ce_bwd(prec, x, c.w, c.bias, c.labels, lse, None, None, x, dw, db, ws, c.B, c.D, c.V)
    within(x, c.dx, c.e_dx, "dx")
    within(dw, c.dw, c.e_dw, "dW")
    within(db, c.db, c.e_db, "db")


@gpu
@pytest.mark.parametrize("shape,prec", [((5, 64, 3000), 0), ((300, 64, 700), 0), ((30, 32, 100), 0), ((300, 65, 700), 1), ((20, 33, 3000), 1)])
def test_linear_ce_off_16_byte_boundaries(binding, shape, prec):
    """Tensors that start anywhere, where rows are not read in place: outputs as well."""
    c = Ce(*shape, prec, True, 0.2, seed=43).reference()

    def off(t):
        return torch.cat([t.flatten()[:1], t.flatten()])[1:].view(t.shape)

    c.x, c.w, c.bias, c.labels = off(c.x), off(c.w), off(c.bias), off(c.labels)
    assert c.x.data_ptr() % 16 and c.w.data_ptr() % 16
    loss, row, lse = c.fwd(binding)
    within(lse, c.lse, c.e_lse, "lse")
    within(row, c.row, c.e_row, "row_loss")
    dx, dw, db = off(torch.full_like(c.x, 7.0)), off(torch.full_like(c.w, 7.0)), off(f32(c.V))
    ws = torch.empty(binding.linear_ce_workspace_bytes(prec, *shape, True), dtype=torch.uint8, device="cuda")
    binding.linear_ce_bwd(prec, c.x, c.w, c.bias, c.labels, lse, None, None, dx, dw, db, ws, *shape)
    within(dx, c.dx, c.e_dx, "dx")
    within(dw, c.dw, c.e_dw, "dW")
    within(db, c.db, c.e_db, "db")


@gpu
def test_linear_ce_two_streams_at_once(binding):
    """Calls that run at the same time, each with a workspace of its own, give what they give alone."""
    pairs = [Ce(300, 72, 9000, 1, True, 0.2, seed=31), Ce(20, 136, 30000, 1, True, 0.2, seed=32), Ce(100, 72, 2000, 0, False, 0.0, seed=33)]
    alone = []
    for c in pairs:
        f = c.fwd(binding)
        alone.append(f + c.bwd(binding, f[2]))
    streams = [torch.cuda.Stream() for _ in pairs]
    torch.cuda.synchronize()
    for _ in range(3):
        together = []
        for c, s in zip(pairs, streams):
            with torch.cuda.stream(s):
                f = c.fwd(binding, s.cuda_stream)
                together.append(f + c.bwd(binding, f[2], stream=s.cuda_stream))
        torch.cuda.synchronize()
        for a, t in zip(alone, together):
            assert all(torch.equal(p, q) for p, q in zip(a, t))


FIRST_CALL_IS_RECORDED = """
import torch
from paper_1804_10574_b200 import binding as b
n, d, v = 300, 64, 500
x, w = torch.randn(n, d, device="cuda").bfloat16(), torch.randn(v, d, device="cuda").bfloat16()
y = torch.randint(0, v, (n,), device="cuda", dtype=torch.int32)
loss, lse, rstd = torch.zeros(1, device="cuda"), torch.zeros(n, device="cuda"), torch.zeros(n, device="cuda")
gamma, h, rng = torch.ones(d, device="cuda").bfloat16(), torch.empty_like(x), torch.zeros(2, dtype=torch.int64, device="cuda")
ws = torch.empty(b.linear_ce_workspace_bytes(1, n, d, v, True), dtype=torch.uint8, device="cuda")
dx, dw, s = torch.empty_like(x), torch.empty_like(w), torch.cuda.Stream()
def step(st):
    b.dropout_fwd(1, x, None, h, rng, n * d, 0.1, 0, st)
    b.add_rmsnorm_fwd(1, h, None, gamma, None, h, None, None, rstd, n, d, 0, 1e-6, st)
    b.linear_ce_fwd(1, h, w, None, y, loss, None, lse, ws, n, d, v, st)
    b.linear_ce_bwd(1, h, w, None, y, lse, None, None, dx, dw, None, ws, n, d, v, False, st)
torch.cuda.synchronize()
g = torch.cuda.CUDAGraph()
with torch.cuda.graph(g, stream=s):
    step(s.cuda_stream)
g.replay()
torch.cuda.synchronize()
a = [t.clone() for t in (loss, lse, dx, dw)]
step(torch.cuda.current_stream().cuda_stream)
torch.cuda.synchronize()
assert all(torch.equal(p, q) for p, q in zip(a, (loss, lse, dx, dw))) and float(loss) > 1
"""


@gpu
def test_first_call_of_a_process_may_be_a_recorded_one(binding):
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    r = subprocess.run([sys.executable, "-c", FIRST_CALL_IS_RECORDED], cwd=root, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stderr[-2000:]


@gpu
def test_offsets_past_32_bits(binding):
    """Tensors of more than 2^31 values: what stands at their ends."""
    C, rows = 16384, 131073 + 64
    x = torch.empty(rows, C, dtype=torch.bfloat16, device="cuda").normal_()
    dy = torch.empty_like(x).normal_()
    y, rstd, gamma = torch.empty_like(x), f32(rows), randn(C, seed=41, prec=1, mean=1.0, std=0.2)
    binding.add_rmsnorm_fwd(1, x, None, gamma, None, y, None, None, rstd, rows, C)
    ends = [0, 1, rows - 2, rows - 1]
    _, r, ref = rms_reference(x[ends], None, gamma, 1e-6)
    within(y[ends], ref, (U[x.dtype] + rms_rel(C) + 2.0 ** -22) * ref.abs(), "y")
    dx, dg = y, f32(C)
    binding.add_rmsnorm_bwd(1, dy, None, x, gamma, rstd, dx, dg, f32(binding.rmsnorm_scratch_elems(rows, C)), rows, C)
    k, g, d = x[ends].double(), gamma.double(), dy[ends].double()
    ref = r[:, None] * (g * d - k * r[:, None] ** 2 * (g * d * k).mean(1, keepdim=True))
    mass = r[:, None] * (g * d).abs() + k.abs() * r[:, None] ** 3 * (g * d * k).abs().mean(1, keepdim=True)
    within(dx[ends], ref, U[x.dtype] * ref.abs() + 40 * 2.0 ** -24 * mass, "dx")
    n = rows * C - 3
    rng = rng_of(5, 6)
    binding.dropout_fwd(1, x, None, y, rng, n, 0.5)
    keep = torch.from_numpy(philox(5, 6 + n // 8 - 100, 0, 102).view(np.uint16).reshape(-1) >= 32768).cuda()
    first = (n // 8 - 100) * 8
    got, src = y.view(-1)[first:n], x.view(-1)[first:n]
    assert torch.equal(got, torch.where(keep[: n - first], src * 2, torch.zeros_like(src)))
    del y, dx
    # the same memory as a projection of 2^31 values and more: few rows and many
    V, D = rows, C
    w = x.mul_(0.01)
    for B in (3, 70):
        c = Ce(B, D, 8, 1, seed=42)
        c.V, c.w = V, w
        c.labels = torch.arange(V - B, V, device="cuda", dtype=torch.int32)
        loss, row, lse = c.fwd(binding)
        parts = torch.cat([c.x.double() @ w[i: i + 8192].double().t() for i in range(0, V, 8192)], 1)
        # 1024 steps of four units of 2^-24 of sums below 16384 x 0.8 x 0.01 x 0.8
        tol = 4 * 1024 * 2.0 ** -24 * 110
        ref = torch.logsumexp(parts, 1)
        within(lse, ref, tol, "lse")
        within(row, ref - parts.gather(1, c.labels.long()[:, None])[:, 0], 2 * tol, "row_loss")
        dw = dy
        ws = torch.empty(binding.linear_ce_workspace_bytes(1, B, D, V, True), dtype=torch.uint8, device="cuda")
        binding.linear_ce_bwd(1, c.x, w, None, c.labels, lse, None, None, None, dw, None, ws, B, D, V)
        dz = (parts[:, -100:] - ref[:, None]).exp()
        dz[torch.arange(B), 100 - B + torch.arange(B)] -= 1.0
        dz /= B
        want, mass = dz.t() @ c.x.double(), dz.abs().t() @ c.x.double().abs()
        within(dw[-100:], want, 2.0 ** -8 * want.abs() + (2.0 ** -8 + 2 * tol) * mass, "dW")


@gpu
def test_linear_ce_leaves_what_it_does_not_own(binding):
    """Buffers with more rows than the call names keep the rows behind the last; inputs are not written."""
    for prec in (0, 1):
        c = Ce(300, 65, 270, prec, True, 0.1, seed=17)
        kept = [t.clone() for t in (c.x, c.w, c.bias, c.labels)]
        n, d, v = 290, 65, 260
        ws_bytes = binding.linear_ce_workspace_bytes(prec, n, d, v, True)
        ws = torch.full((ws_bytes + 4096,), 77, dtype=torch.uint8, device="cuda")
        loss, row, lse = f32(1), f32(300), f32(300)
        dx, dw, db = torch.full_like(c.x, 7.0), torch.full_like(c.w, 7.0), f32(270)
        fws = torch.full((binding.linear_ce_workspace_bytes(prec, n, d, v, False),), 255, dtype=torch.uint8, device="cuda")
        binding.linear_ce_fwd(prec, c.x, c.w, c.bias, c.labels, loss, row, lse, fws, n, d, v)
        binding.linear_ce_bwd(prec, c.x, c.w, c.bias, c.labels, lse, None, None, dx, dw, db, ws[:ws_bytes], n, d, v)
        torch.cuda.synchronize()
        assert (row[n:] == 7).all() and (lse[n:] == 7).all() and (dx[n:] == 7).all() and (dw[v:] == 7).all() and (db[v:] == 7).all()
        assert (ws[ws_bytes:] == 77).all()
        assert all(torch.equal(a, b) for a, b in zip(kept, (c.x, c.w, c.bias, c.labels)))


@gpu
def test_linear_ce_refuses_on_the_gpu(binding):
    c = Ce(4, 64, 100, 1, seed=18)
    ws = torch.empty(binding.linear_ce_workspace_bytes(1, 4, 64, 100, False) + 512, dtype=torch.uint8, device="cuda")
    row = f32(4)

    def call(x=c.x, labels=c.labels, w=c.w, ws=ws, row=row):
        binding.linear_ce_fwd(1, x, w, None, labels, None, row, None, ws, 4, 64, 100)

    call()
    for kw in ({"x": c.x.data_ptr() + 2}, {"ws": ws[:512]}, {"ws": ws[8:]}, {"labels": c.labels.cpu()}, {"row": row.cpu()}):
        with pytest.raises(binding.DdgError) as e:
            call(**kw)
        assert e.value.status == 1
    for kw in ({"x": c.x.float()}, {"x": c.x.half()}, {"w": c.w.t()}, {"labels": c.labels.long()}, {"labels": c.labels.float()}, {"row": row[:3]}):
        with pytest.raises(ValueError):
            call(**kw)
    torch.cuda.synchronize()


# ---- RMS norm -------------------------------------------------------------------------------------------------------
RMS_SHAPES = [(1, 1), (1, 8), (3, 7), (5, 64), (7, 128), (2, 1000), (9, 1021), (33, 1024), (130, 2048), (4, 4096), (700, 136), (3, 5000),
              (2, 8192), (3, 16384), (2, 16383), (1300, 40)]


def rms_inputs(rows, C, prec, seed):
    return (randn(rows, C, seed=seed, prec=prec), randn(rows, C, seed=seed + 1, prec=prec, std=3.0),
            randn(C, seed=seed + 2, prec=prec, std=0.2, mean=1.0))


def rms_reference(x, res, gamma, eps):
    h = x.double() + (res.double() if res is not None else 0.0)
    rstd = 1.0 / (h.square().mean(1) + eps).sqrt()
    return h, rstd, h * rstd[:, None] * gamma.double()


def rms_rel(C):
    """Relative error of rstd and, above it, of y in 32 bits: a sum of squares over at most 16 values per thread and a
    tree of 10 steps (half of it after the root), the addition, the division, rsqrt (2 steps)."""
    return (13 + 6) * 2.0 ** -24


@gpu
@PREC
@pytest.mark.parametrize("shape", RMS_SHAPES, ids=lambda s: "x".join(map(str, s)))
def test_add_rmsnorm_forward(binding, shape, prec):
    rows, C = shape
    x, res, gamma = rms_inputs(rows, C, prec, 21)
    for r in (res, None):
        h, y, rstd = torch.full_like(x, 7.0), torch.full_like(x, 7.0), f32(rows)
        binding.add_rmsnorm_fwd(prec, x, r, gamma, h if r is not None else None, y, None, None, rstd, rows, C)
        h_ref, rstd_ref, y_ref = rms_reference(x, r, gamma, 1e-6)
        u, e = U[x.dtype], rms_rel(C) + 2.0 ** -23
        if r is not None:
            within(h, h_ref, u * h_ref.abs() + 2.0 ** -24 * h_ref.abs(), "h")
        within(rstd, rstd_ref, e * rstd_ref, "rstd")
        within(y, y_ref, (u + e + 2.0 ** -22) * y_ref.abs() + 1e-37, "y")


@gpu
@PREC
@pytest.mark.parametrize("group", [0, 128])
@pytest.mark.parametrize("shape", [(1, 128), (5, 4096), (300, 512), (2, 16384), (3, 1021), (1, 1), (17, 2944)], ids=lambda s: "x".join(map(str, s)))
def test_add_rmsnorm_to_8_bits(binding, shape, prec, group):
    """Scales against the reference's; the stored values within half a step of e4m3 (2^-4 of the value, 2^-10 below the
    smallest normal one) of y / scale, and y and q from one call."""
    rows, C = shape
    if group and C % group:
        pytest.skip("no whole groups")
    x, res, gamma = rms_inputs(rows, C, prec, 31)
    x[0, : min(C, 128)] = 0.0
    res[0, : min(C, 128)] = 0.0  # a group of zeros, a row of them where that is all
    h, y = torch.full_like(x, 7.0), torch.full_like(x, 7.0)
    q, scale = torch.empty(rows, C, dtype=torch.float8_e4m3fn, device="cuda"), f32(rows, C // (group or C))
    binding.add_rmsnorm_fwd(prec, x, res, gamma, h, y, q, scale, None, rows, C, group)
    _, _, y_ref = rms_reference(x, res, gamma, 1e-6)
    blocks = y_ref.view(rows, -1, group or C)
    top = blocks.abs().amax(2)
    s_ref = torch.where(top > 0, top / 448.0, 1.0)
    e = rms_rel(C) + 2.0 ** -21
    within(scale, s_ref, e * s_ref, "scale")
    within(y, y_ref, (U[x.dtype] + e) * y_ref.abs(), "y")
    got = q.double().view_as(blocks) * scale.double()[..., None]
    within(got, blocks, (2.0 ** -4 + 2 * e) * blocks.abs() + 2.0 ** -10 * s_ref[..., None] * 1.01, "q")
    assert float(q.float().abs().max()) == 448.0 or not y_ref.any()
    q2, scale2 = torch.empty_like(q), torch.empty_like(scale)
    binding.add_rmsnorm_fwd(prec, x, res, gamma, h, None, q2, scale2, None, rows, C, group)
    assert torch.equal(q.view(torch.uint8), q2.view(torch.uint8)) and torch.equal(scale, scale2)


@gpu
@PREC
@pytest.mark.parametrize("shape", RMS_SHAPES, ids=lambda s: "x".join(map(str, s)))
def test_add_rmsnorm_backward(binding, shape, prec):
    rows, C = shape
    h, dh, gamma = rms_inputs(rows, C, prec, 41)
    dy = randn(rows, C, seed=44, prec=prec)
    rstd = (1.0 / (h.double().square().mean(1) + 1e-6).sqrt()).float()
    for extra in (dh, None):
        dx, dgamma = torch.full_like(h, 7.0), f32(C)
        scratch = f32(binding.rmsnorm_scratch_elems(rows, C), fill=NAN)
        binding.add_rmsnorm_bwd(prec, dy, extra, h, gamma, rstd, dx, dgamma, scratch, rows, C)
        r, k, g, d = rstd.double()[:, None], h.double(), gamma.double(), dy.double()
        dot = (g * d * k).mean(1, keepdim=True)
        add = extra.double() if extra is not None else torch.zeros_like(k)
        ref = add + r * (g * d - k * r * r * dot)
        # products and their sum (at most 16 per thread, a tree), then four roundings of every term
        e = (16 + 10 + 6) * 2.0 ** -24
        mass = add.abs() + r * (g * d).abs() + (k * r ** 3).abs() * (g * d * k).abs().mean(1, keepdim=True)
        within(dx, ref, U[h.dtype] * ref.abs() + e * mass, "dx")
        dg, dg_mass = (d * k * r).sum(0), (d * k * r).abs().sum(0)
        # rows / walkers + walkers / 16 + 16 additions
        within(dgamma, dg, (math.ceil(rows / 592) + 37 + 16 + 3) * 2.0 ** -24 * dg_mass, "dgamma")


@gpu
@PREC
def test_add_rmsnorm_special_rows(binding, prec):
    """A row of zeros, of NaN, with an infinity: each row its own."""
    rows, C = 6, 256
    x, res, gamma = rms_inputs(rows, C, prec, 51)
    x[1], res[1] = 0.0, 0.0
    x[2, 7], x[3, 9] = NAN, INF
    h, y, q, scale, rstd = torch.empty_like(x), torch.empty_like(x), torch.empty(rows, C, dtype=torch.float8_e4m3fn, device="cuda"), f32(rows), f32(rows)
    binding.add_rmsnorm_fwd(prec, x, res, gamma, h, y, q, scale, rstd, rows, C)
    assert not y[1].any() and float(scale[1]) == 1.0 and not q[1].float().any() and float(rstd[1]) == pytest.approx(1000.0)
    assert torch.isnan(y[2]).all() and torch.isnan(q[2].float()).all()
    assert float(rstd[3]) == 0.0 and torch.isnan(y[3, 9]) and not y[3, :9].any()
    for r in (0, 4, 5):
        assert torch.isfinite(y[r].float()).all() and torch.isfinite(q[r].float()).all()


@gpu
@PREC
@pytest.mark.parametrize("group", [0, 128])
@pytest.mark.parametrize("gain", [2.0 ** -120, 2.0 ** -130])
def test_add_rmsnorm_to_8_bits_of_tiny_values(binding, prec, group, gain):
    """Values whose maximum over 448 is below the smallest normal number: the scale stops at 2^-126, a power of two, so
    that y / scale is off by the rounding of y alone (2^-150 at least) before it is rounded to e4m3."""
    rows, C = 5, 256
    x, res, gamma = rms_inputs(rows, C, prec, 33)
    gamma.fill_(gain)
    h, y = torch.empty_like(x), torch.empty_like(x)
    q, scale = torch.empty(rows, C, dtype=torch.float8_e4m3fn, device="cuda"), f32(rows, C // (group or C))
    binding.add_rmsnorm_fwd(prec, x, res, gamma, h, y, q, scale, None, rows, C, group)
    _, _, y_ref = rms_reference(x, res, gamma, 1e-6)
    assert float(y_ref.abs().max()) < 448 * 2.0 ** -126
    assert (scale == 2.0 ** -126).all()
    e = rms_rel(C) + 2.0 ** -22
    within(q.double() * 2.0 ** -126, y_ref, (2.0 ** -4 + 2 * e) * y_ref.abs() + 2.0 ** -10 * 2.0 ** -126 + 2.0 ** -150, "q")


@gpu
@PREC
@pytest.mark.parametrize("C", [4096, 1021])
def test_add_rmsnorm_in_place(binding, prec, C):
    """h over x or res, y over x, dx over dy, dh or h: the same bits as into buffers of their own."""
    rows = 19
    x, res, gamma = rms_inputs(rows, C, prec, 61)
    h, y, rstd = torch.empty_like(x), torch.empty_like(x), f32(rows)
    binding.add_rmsnorm_fwd(prec, x, res, gamma, h, y, None, None, rstd, rows, C)
    a, b = x.clone(), res.clone()
    binding.add_rmsnorm_fwd(prec, a, b, gamma, b, a, None, None, None, rows, C)
    assert torch.equal(a, y) and torch.equal(b, h)
    dy, dg, scratch = randn(rows, C, seed=64, prec=prec), f32(C), f32(binding.rmsnorm_scratch_elems(rows, C))
    dx = torch.empty_like(x)
    binding.add_rmsnorm_bwd(prec, dy, res, h, gamma, rstd, dx, dg, scratch, rows, C)
    for k in range(3):
        t = [dy.clone(), res.clone(), h.clone()]
        binding.add_rmsnorm_bwd(prec, t[0], t[1], t[2], gamma, rstd, t[k], dg, scratch, rows, C)
        assert torch.equal(t[k], dx), k


@gpu
@PREC
def test_add_rmsnorm_off_16_byte_boundaries(binding, prec):
    """Tensors that start anywhere give the aligned ones' results; only scales per group need the boundary."""
    rows, C = 5, 512
    x, res, gamma = rms_inputs(rows, C, prec, 71)
    y, y2 = torch.empty_like(x), torch.empty(rows * C + 1, dtype=x.dtype, device="cuda")[1:].view(rows, C)
    h = torch.empty_like(x)
    binding.add_rmsnorm_fwd(prec, x, res, gamma, h, y, None, None, None, rows, C)
    off = [torch.cat([t.flatten()[:1], t.flatten()])[1:].view(t.shape) for t in (x, res, gamma)]
    assert off[0].data_ptr() % 16
    binding.add_rmsnorm_fwd(prec, *off, torch.empty_like(x), y2, None, None, None, rows, C)
    _, _, ref = rms_reference(x, res, gamma, 1e-6)
    within(y2, ref, (U[x.dtype] + rms_rel(C) + 2.0 ** -22) * ref.abs(), "y")
    with pytest.raises(binding.DdgError) as e:
        binding.add_rmsnorm_fwd(prec, *off, torch.empty_like(x), None, torch.empty(rows, C, dtype=torch.uint8, device="cuda"), f32(rows, 4), None, rows, C, 128)
    assert e.value.status == 1


@gpu
def test_add_rmsnorm_gradient_against_differences(binding):
    rows, C = 12, 96
    x, res, gamma = rms_inputs(rows, C, 0, 81)
    dy = randn(rows, C, seed=84, prec=0)
    dh = randn(rows, C, seed=85, prec=0)

    def value(x, gamma):
        h, y = torch.empty_like(x), torch.empty_like(x)
        binding.add_rmsnorm_fwd(0, x, res, gamma, h, y, None, None, None, rows, C)
        return float((y.double() * dy.double()).sum() + (h.double() * dh.double()).sum())

    h, y, rstd, dx, dg = torch.empty_like(x), torch.empty_like(x), f32(rows), torch.empty_like(x), f32(C)
    binding.add_rmsnorm_fwd(0, x, res, gamma, h, y, None, None, rstd, rows, C)
    binding.add_rmsnorm_bwd(0, dy, dh, h, gamma, rstd, dx, dg, f32(binding.rmsnorm_scratch_elems(rows, C)), rows, C)
    step = 2.0 ** -4
    for t, grad in ((x, dx), (gamma, dg)):
        d = randn(*t.shape, seed=86, prec=0)
        d /= d.norm()
        args = [(t + s * d, gamma) if t is x else (x, t + s * d) for s in (step, -step)]
        slope, want = (value(*args[0]) - value(*args[1])) / (2 * step), float((grad.double() * d.double()).sum())
        # values: about sqrt(1152) sums of terms rounded to 2^-22; third derivative: |dy| rstd^3 along a unit direction
        assert abs(slope - want) < 1152 * 3 * 2.0 ** -22 / step + step ** 2 / 6 * 6 * 40 * 0.05, (slope, want)


# ---- dropout --------------------------------------------------------------------------------------------------------
def philox(key, counter, layer, count):
    """Philox4x32-10, plain integers."""
    out = np.empty((count, 4), dtype=np.uint32)
    for i in range(count):
        at = (counter + i) % 2 ** 64
        c, k = [at % 2 ** 32, at >> 32, layer, 0], [key % 2 ** 32, key >> 32]
        for _ in range(10):
            p, q = c[0] * 0xD2511F53, c[2] * 0xCD9E8D57
            c = [(q >> 32) ^ c[1] ^ k[0], q % 2 ** 32, (p >> 32) ^ c[3] ^ k[1], p % 2 ** 32]
            k = [(k[0] + 0x9E3779B9) % 2 ** 32, (k[1] + 0xBB67AE85) % 2 ** 32]
        out[i] = c
    return out


def keep_mask(key, counter, layer, n, p):
    return (philox(key, counter, layer, -(-n // 8)).view(np.uint16).reshape(-1)[:n] >= round(p * 65536))


def rng_of(key, counter):
    return torch.from_numpy(np.array([key, counter], dtype=np.uint64).view(np.int64)).cuda()


def test_philox_of_this_file_gives_the_published_numbers():
    """The known answers for counter and key of zeros and of ones (Salmon et al., 2011)."""
    assert [hex(v) for v in philox(0, 0, 0, 1)[0].tolist()] == ["0x6627e8d5", "0xe169c58d", "0xbc57ac4c", "0x9b00dbd8"]


@gpu
@PREC
@pytest.mark.parametrize("n", [1, 7, 8, 9, 255, 4096, 20011])
@pytest.mark.parametrize("p", [0.0, 0.1, 0.5, 1.0])
def test_dropout(binding, n, p, prec):
    """Every element against the generator's definition; positions that pass 32 and 64 bits; a layer of its own."""
    for key, counter, layer in ((0, 0, 0), (0x123456789ABCDEF0, 2 ** 32 - 3, 5), (2 ** 64 - 1, 2 ** 64 - 2, 2 ** 32 - 1)):
        keep = torch.from_numpy(keep_mask(key, counter, layer, n, p)).cuda()
        x, res, rng = randn(n, seed=91, prec=prec), randn(n, seed=92, prec=prec), rng_of(key, counter)
        scale = 65536 / (65536 - round(p * 65536)) if p < 1 else 0.0
        for r in (res, None):
            y = torch.full_like(x, 7.0)
            binding.dropout_fwd(prec, x, r, y, rng, n, p, layer)
            kept = torch.where(keep, x.double() * scale, 0.0)
            ref = kept + (r.double() if r is not None else 0.0)
            within(y, ref, U[x.dtype] * ref.abs() + 3 * 2.0 ** -24 * (kept.abs() + ref.abs()), "y")
        dx = torch.full_like(x, 7.0)
        binding.dropout_bwd(prec, x, dx, rng, n, p, layer)
        assert torch.equal(dx, y), "the backward pass is the forward pass without a residual"


@gpu
@PREC
def test_dropout_special_values_in_place_and_unaligned(binding, prec):
    n, p, rng = 1003, 0.5, rng_of(3, 4)
    keep = torch.from_numpy(keep_mask(3, 4, 0, n, p)).cuda()
    x, res = torch.full((n,), NAN, device="cuda", dtype=DT[prec]), randn(n, seed=93, prec=prec)
    y = torch.empty_like(x)
    binding.dropout_fwd(prec, x, res, y, rng, n, p)
    assert torch.isnan(y[keep]).all() and torch.equal(y[~keep], res[~keep])
    x = randn(n, seed=94, prec=prec)
    binding.dropout_fwd(prec, x, res, y, rng, n, p)
    for k in range(2):
        t = [x.clone(), res.clone()]
        binding.dropout_fwd(prec, t[0], t[1], t[k], rng, n, p)
        assert torch.equal(t[k], y), k
    off = torch.full((n + 2,), 7.0, device="cuda", dtype=DT[prec])
    binding.dropout_fwd(prec, x, res, off[1:], rng, n, p)
    assert torch.equal(off[1:-1], y) and float(off[0]) == 7.0 and float(off[-1]) == 7.0


@gpu
def test_dropout_share_and_recorded_positions(binding):
    """The share of dropped values (four standard deviations); a recorded call draws new numbers when the position in
    device memory moved on, and the old ones when it went back."""
    n, p = 1 << 20, 0.3
    x, y, rng = torch.ones(n, device="cuda"), torch.empty(n, device="cuda"), rng_of(7, 0)
    stream = torch.cuda.Stream()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        binding.dropout_fwd(0, x, None, y, rng, n, p, 0, torch.cuda.current_stream().cuda_stream)
    seen = []
    for at in (0, n // 8, 0):
        rng[1] = at
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        seen.append(y.clone())
        share = float((y == 0).double().mean())
        t = round(p * 65536) / 65536
        assert abs(share - t) < 4 * math.sqrt(t * (1 - t) / n)
    assert torch.equal(seen[0], seen[2]) and not torch.equal(seen[0], seen[1])
    both = (seen[0] == 0) & (seen[1] == 0)
    assert abs(float(both.double().mean()) - t * t) < 4 * math.sqrt(t * t * (1 - t * t) / n)


# ---- the three in a row ---------------------------------------------------------------------------------------------
@gpu
def test_tail_of_a_training_step(binding):
    """dropout + residual -> RMS norm -> projection and loss, and all of it backwards and into the update, in 32 bits,
    against automatic differentiation of the formulas in 64."""
    n, d, v, p, eps, lr = 200, 96, 700, 0.25, 1e-5, 0.5
    x, res, gamma = randn(n, d, seed=101, prec=0), randn(n, d, seed=102, prec=0), randn(d, seed=103, prec=0, std=0.2, mean=1.0)
    w = randn(v, d, seed=104, prec=0, std=0.2)
    labels = torch.randint(0, v, (n,), device="cuda", dtype=torch.int32)
    labels[::7] = -1
    rng = rng_of(11, 12)
    h, y, rstd = torch.empty_like(x), torch.empty_like(x), f32(n)
    loss, lse = f32(1), f32(n)
    ws = torch.empty(max(binding.linear_ce_workspace_bytes(0, n, d, v, k) for k in (0, 1)), dtype=torch.uint8, device="cuda")
    binding.dropout_fwd(0, x, res, h, rng, n * d, p)
    binding.add_rmsnorm_fwd(0, h, None, gamma, None, y, None, None, rstd, n, d, 0, eps)
    binding.linear_ce_fwd(0, y, w, None, labels, loss, None, lse, ws, n, d, v)
    dy, dw, dh, dgamma, dx = torch.empty_like(x), torch.empty_like(w), torch.empty_like(x), f32(d), torch.empty_like(x)
    binding.linear_ce_bwd(0, y, w, None, labels, lse, None, None, dy, dw, None, ws, n, d, v, True)
    binding.add_rmsnorm_bwd(0, dy, None, h, gamma, rstd, dh, dgamma, f32(binding.rmsnorm_scratch_elems(n, d)), n, d)
    binding.dropout_bwd(0, dh, dx, rng, n * d, p)
    w_new, mom, version = w.clone(), torch.zeros_like(w), torch.empty_like(w)
    binding.sgd_update(0, w_new, mom, dw, version, v * d, lr, 0.0, 0.0)
    keep = torch.from_numpy(keep_mask(11, 12, 0, n * d, p)).cuda().view(n, d)
    leaves = [t.double().requires_grad_() for t in (x, res, gamma, w)]
    X, R, G, W = leaves
    hh = R + torch.where(keep, X / (1 - p), 0.0)
    yy = hh * torch.rsqrt(hh.square().mean(1, keepdim=True) + eps) * G
    z = yy @ W.t()
    counted = labels >= 0
    ref = (torch.logsumexp(z, 1) - z.gather(1, labels.clamp(min=0).long()[:, None])[:, 0])[counted].mean()
    ref.backward()
    # the longest way to a gradient: 6 x 6 steps of the projection's accumulator (four units each), 6 x 44 of the gradient's,
    # and under 100 single roundings; every step relative to sums of absolute values, which exceed the sums' norm by less
    # than a factor sqrt(700)
    tol = (4 * (36 + 264) + 100) * 2.0 ** -24 * math.sqrt(700)
    assert abs(float(loss[0]) - float(ref.detach())) < 2.0 ** -16 * float(ref.detach())
    for got, leaf, name in ((dx, X, "x"), (dh, R, "res"), (dgamma, G, "gamma"), (dw, W, "w")):
        assert float((got.double() - leaf.grad).norm() / leaf.grad.norm()) < tol, name
    assert torch.equal(version, w_new)
    within(w_new, W.detach() - lr * W.grad, lr * tol * W.grad.norm() + 2.0 ** -23 * W.detach().abs(), "the updated projection")


# ---- refusals without a GPU -----------------------------------------------------------------------------------------
def status(fn, *args):
    from paper_1804_10574_b200 import binding as b
    with pytest.raises(b.DdgError) as e:
        fn(*args)
    return e.value.status


P = 1 << 20  # an address that no refused call looks at


class Ws:
    """A workspace of a size of its own at that address."""

    def __init__(self, n, at=P):
        self.n, self.at = n, at

    def numel(self):
        return self.n

    def element_size(self):
        return 1

    def data_ptr(self):
        return self.at


def test_linear_ce_refusals(binding):
    need = binding.linear_ce_workspace_bytes(1, 4, 64, 100, False)
    assert need > 0 and binding.linear_ce_workspace_bytes(1, 4, 64, 100, True) > 0
    for bad in ((2, 4, 64, 100), (1, 0, 64, 100), (1, 4, 0, 100), (1, 4, 64, 0), (1, 4, 64, (1 << 24) + 1)):
        assert binding.linear_ce_workspace_bytes(*bad, False) == 0
    ok = dict(prec=1, x=P, W=P, bias=None, labels=P, loss=P, row_loss=P, lse=P, ws=Ws(need), B=4, n_in=64, n_out=100)
    fwd = lambda **kw: status(binding.linear_ce_fwd, *{**ok, **kw}.values())  # noqa: E731
    assert fwd(prec=2) == 1 and fwd(prec=-1) == 1
    for name in ("x", "W", "labels", "ws"):
        assert fwd(**{name: None}) == 1
    assert fwd(loss=None, row_loss=None, lse=None) == 1
    for name in ("B", "n_in", "n_out"):
        assert fwd(**{name: 0}) == 3 and fwd(**{name: -5}) == 3 and fwd(**{name: 1 << 25}) == 3
    assert fwd(x=P + 2) == 1 and fwd(W=P + 8) == 1                 # read in place: 16-byte boundaries
    assert fwd(ws=Ws(need - 1)) == 1 and fwd(ws=Ws(need, P + 16)) == 1
    assert b"workspace" in binding.lib().ddg_last_error(None)
    need = binding.linear_ce_workspace_bytes(1, 4, 64, 100, True)
    okb = dict(prec=1, x=P, W=P, bias=None, labels=P, lse=P, dloss=None, drow=None, dx=P, dW=2 * P, db=None, ws=Ws(need), B=4, n_in=64, n_out=100)
    bwd = lambda **kw: status(binding.linear_ce_bwd, *{**okb, **kw}.values())  # noqa: E731
    for name in ("x", "W", "labels", "lse", "ws"):
        assert bwd(**{name: None}) == 1
    assert bwd(dx=None, dW=None) == 1 and bwd(dloss=P, drow=P) == 1
    assert bwd(W=P, dW=P) == 1                                     # the projection is read after its first gradients are written
    assert bwd(B=0) == 3 and bwd(ws=Ws(need - 1)) == 1 and bwd(prec=7) == 1


def test_rmsnorm_refusals(binding):
    ok = dict(prec=1, x=P, res=P, gamma=P, h=P, y=P, y8=None, s8=None, rstd=None, rows=3, C=256, group=0, eps=1e-6)
    fwd = lambda **kw: status(binding.add_rmsnorm_fwd, *{**ok, **kw}.values())  # noqa: E731
    assert fwd(prec=3) == 1 and fwd(x=None) == 1 and fwd(gamma=None) == 1 and fwd(y=None) == 1 and fwd(h=None) == 1
    assert fwd(y8=P) == 1 and fwd(s8=P) == 1                       # values and scales come together
    assert fwd(eps=-1.0) == 1 and fwd(eps=NAN) == 1 and fwd(eps=INF) == 1
    assert fwd(group=64) == 1 and fwd(y8=P, s8=P, group=128, C=200) == 3 and fwd(y8=P, s8=P, group=128, x=P + 2) == 1
    assert fwd(rows=0) == 3 and fwd(C=0) == 3 and fwd(C=16385) == 3 and fwd(rows=(1 << 30) + 1) == 3
    okb = dict(prec=1, dy=P, dh=None, h=P, gamma=P, rstd=P, dx=P, dgamma=P, scratch=P, rows=3, C=256)
    bwd = lambda **kw: status(binding.add_rmsnorm_bwd, *{**okb, **kw}.values())  # noqa: E731
    for name in ("dy", "h", "gamma", "rstd", "dx", "dgamma", "scratch"):
        assert bwd(**{name: None}) == 1
    assert bwd(rows=0) == 3 and bwd(C=16385) == 3
    assert binding.rmsnorm_scratch_elems(0, 8) == 0 and binding.rmsnorm_scratch_elems(2, 16385) == 0 and binding.rmsnorm_scratch_elems(2, 8) > 0


def test_dropout_refusals(binding):
    ok = dict(prec=1, x=P, res=None, y=P, rng=P, n=8, p=0.1)
    fwd = lambda **kw: status(binding.dropout_fwd, *{**ok, **kw}.values())  # noqa: E731
    assert fwd(prec=9) == 1 and fwd(x=None) == 1 and fwd(y=None) == 1 and fwd(rng=None) == 1
    assert fwd(p=-0.1) == 1 and fwd(p=1.5) == 1 and fwd(p=NAN) == 1 and fwd(rng=P + 4) == 1 and fwd(n=0) == 3
    assert status(binding.dropout_bwd, 1, None, P, P, 8, 0.1) == 1


@gpu
@PREC
@pytest.mark.parametrize("shape", [(1, 2), (9, 3), (3, 9), (70, 33), (2000, 129), (300, 517), (1500, 1023), (40, 8191), (700, 8189), (20, 12289), (5, 16383)], ids=lambda s: "x".join(map(str, s)))
def test_add_rmsnorm_of_odd_widths(binding, prec, shape):
    """Rows that start anywhere: forward, to 8 bits and backward, in buffers between guards and in place."""
    rows, C = shape
    x, res, gamma = rms_inputs(rows, C, prec, 101)
    dh, dy = randn(rows, C, seed=104, prec=prec), randn(rows, C, seed=105, prec=prec)
    guard = 64

    def guarded(dtype):
        t = torch.zeros(rows * C + guard, dtype=torch.float32, device="cuda").to(dtype)
        t[rows * C:] = 3.0
        return t, t[: rows * C].view(rows, C)

    bufs = [guarded(x.dtype) for _ in range(3)] + [guarded(torch.float8_e4m3fn)]
    h, y, dx, q = (b[1] for b in bufs)
    scale, rstd = f32(rows), f32(rows)
    binding.add_rmsnorm_fwd(prec, x, res, gamma, h, y, q, scale, rstd, rows, C)
    h_ref, rstd_ref, y_ref = rms_reference(x, res, gamma, 1e-6)
    e = rms_rel(C) + 2.0 ** -21
    within(h, h_ref, (U[x.dtype] + 2.0 ** -24) * h_ref.abs(), "h")
    within(rstd, rstd_ref, e * rstd_ref, "rstd")
    # h itself is off by its sum's rounding, 2^-24 of it
    within(y, y_ref, (U[x.dtype] + e) * y_ref.abs() + 1e-37, "y")
    s_ref = y_ref.abs().amax(1) / 448.0
    within(scale, s_ref, e * s_ref, "scale")
    within(q.double() * scale.double()[:, None], y_ref, (2.0 ** -4 + 2 * e) * y_ref.abs() + 2.0 ** -10 * s_ref[:, None] * 1.01, "q")
    dgamma, scratch = f32(C), f32(binding.rmsnorm_scratch_elems(rows, C), fill=NAN)
    binding.add_rmsnorm_bwd(prec, dy, dh, h, gamma, rstd, dx, dgamma, scratch, rows, C)
    r, k, g, d = rstd.double()[:, None], h.double(), gamma.double(), dy.double()
    ref = dh.double() + r * (g * d - k * r * r * (g * d * k).mean(1, keepdim=True))
    mass = dh.double().abs() + r * (g * d).abs() + (k * r ** 3).abs() * (g * d * k).abs().mean(1, keepdim=True)
    # at most 32 products per thread, a tree over 1024 threads, then four roundings of every term
    within(dx, ref, U[x.dtype] * ref.abs() + (32 + 10 + 6) * 2.0 ** -24 * mass, "dx")
    dg, dg_mass = (d * k * r).sum(0), (d * k * r).abs().sum(0)
    # at least 144 walkers of at most 888 in the fold, two roundings of a product
    within(dgamma, dg, (math.ceil(rows / 144) + 888 / 32 + 32 + 3) * 2.0 ** -24 * dg_mass, "dgamma")
    for t, _ in bufs:
        assert (t[rows * C:].float() == 3.0).all()
    a, b = x.clone(), res.clone()
    binding.add_rmsnorm_fwd(prec, a, b, gamma, b, a, None, None, None, rows, C)
    assert torch.equal(a, y) and torch.equal(b, h)
    for j in range(3):
        t = [dy.clone(), dh.clone(), h.clone()]
        binding.add_rmsnorm_bwd(prec, t[0], t[1], t[2], gamma, rstd, t[j], dgamma, scratch, rows, C)
        assert torch.equal(t[j], dx), j


def test_workspace_has_to_be_contiguous(binding):
    """Its length is counted from its elements, which an expanded tensor does not have."""
    x, ws = torch.zeros(4, 8), torch.zeros(1, dtype=torch.uint8).expand(1 << 20)
    with pytest.raises(ValueError):
        binding.linear_ce_fwd(0, x, x, None, torch.zeros(4, dtype=torch.int32), torch.zeros(1), None, None, ws, 4, 8, 4)


@gpu
@pytest.mark.parametrize("shape", [(2000, 4096), (2000, 512), (40, 4096)], ids=lambda s: "x".join(map(str, s)))
def test_add_rmsnorm_backward_scratch_at_any_16_byte_boundary(binding, shape):
    rows, C = shape
    h, dh, gamma = rms_inputs(rows, C, 1, 91)
    dy, rstd = randn(rows, C, seed=94, prec=1), f32(rows, fill=0.3)
    n = binding.rmsnorm_scratch_elems(rows, C)
    got = []
    for skip in (0, 4, 1):
        dx, dgamma = torch.empty_like(h), f32(C)
        scratch = f32(n + skip)[skip:]
        binding.add_rmsnorm_bwd(1, dy, dh, h, gamma, rstd, dx, dgamma, scratch, rows, C)
        got.append((dx, dgamma))
    assert torch.equal(got[0][0], got[1][0]) and torch.equal(got[0][1], got[1][1])
    # off 16 bytes the sums are split over the threads in another way
    d, k, r = dy.double(), h.double(), rstd.double()[:, None]
    bound = 2 * (math.ceil(rows / 148) + 37 + 16 + 3) * 2.0 ** -24 * (d * k * r).abs().sum(0)
    within(got[2][1], got[0][1].double(), bound, "dgamma")


def test_tensor_arguments_are_checked_in_the_binding(binding):
    """What a C call cannot see: strides, types and lengths of the tensors behind the addresses."""
    x = torch.zeros(4, 8)
    for bad in (x.t(), x.half(), x[:2]):
        with pytest.raises(ValueError):
            binding.dropout_fwd(0, bad, None, P, P, 32, 0.1)


WAITS_RUN_OUT = """
import torch
from paper_1804_10574_b200 import binding as b
for prec, n, d, v in ((1, 300, 136, 3000), (1, 700, 2200, 1100), (0, 300, 136, 700), (1, 8200, 64, 17000), (1, 1, 2048, 9000), (1, 20, 136, 3001), (1, 64, 2048, 12000)):
    dt = torch.bfloat16 if prec else torch.float32
    x, w = torch.randn(n, d, device="cuda").to(dt), torch.randn(v, d, device="cuda").to(dt)
    y = torch.randint(0, v, (n,), device="cuda", dtype=torch.int32)
    out = [torch.zeros(k, device="cuda") for k in (1, n, n)] + [torch.empty_like(x), torch.empty_like(w), torch.zeros(v, device="cuda")]
    ws = torch.empty(max(b.linear_ce_workspace_bytes(prec, n, d, v, k) for k in (0, 1)), dtype=torch.uint8, device="cuda")
    for polls in (1, 2, 3, 5, 9, 17, 40, 200, 0):
        b.debug_linear_ce_wait_polls(polls)
        b.linear_ce_fwd(prec, x, w, None, y, out[0], out[1], out[2], ws, n, d, v)
        b.linear_ce_bwd(prec, x, w, None, y, out[2], None, None, out[3], out[4], out[5], ws, n, d, v)
        torch.cuda.synchronize()
    assert all(bool(torch.isnan(t).all()) for t in out[:3])
    assert float((torch.ones(8, device="cuda") * 2).sum()) == 16.0
"""


@gpu
def test_linear_ce_waits_that_run_out_end_cleanly(binding):
    """Waits with limits of few polls and of none, at every way that waits on the device: each kernel lets its copies and products
    land, frees its tensor memory and returns; the forward pass's results are NaN.  In a process of its own."""
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    r = subprocess.run([sys.executable, "-c", WAITS_RUN_OUT], cwd=root, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stderr[-2000:]


# every way of a call that waits on the device: rows with one chunk, with a K range that is cut, with splits, fp32, several chunks,
# 16 / 32 / 64 rows
WAYS_THAT_WAIT = [(300, 136, 777, 1), (700, 2200, 1100, 1), (2100, 264, 9000, 1), (300, 136, 700, 0), (8200, 40, 17000, 1), (1, 2048, 9000, 1), (20, 136, 3001, 1), (64, 2048, 12000, 1)]


@gpu
@pytest.mark.parametrize("shape", WAYS_THAT_WAIT, ids=lambda s: "x".join(map(str, s)))
def test_linear_ce_results_of_a_call_whose_wait_ran_out_are_nan(binding, shape):
    """All results of that call, whichever are asked for; with a limit that its waits keep, they are the usual bits; the
    calls after it are not touched."""
    c = Ce(*shape, bias=True, ignored=0.1, seed=51)
    fwd = c.fwd(binding)
    lse = fwd[2]
    wants = [("xwb", False), ("x", False), ("w", True), ("b", False)]
    bwd = [[t for t in c.bwd(binding, lse, want=w, dw_f32=f) if t is not None] for w, f in wants]
    try:
        for polls in (0, 1, 2, 1, 4, 1, 8, 16, 50, 400, 0):
            binding.debug_linear_ce_wait_polls(polls)
            got = [c.fwd(binding)] + [[t for t in c.bwd(binding, lse, want=w, dw_f32=f) if t is not None] for w, f in wants]
            torch.cuda.synchronize()
            for g, ref in zip(got, [fwd] + bwd):
                failed = bool(torch.isnan(g[0].flatten()[0]))
                assert failed or polls > 0
                for a, b in zip(g, ref):
                    assert bool(torch.isnan(a).all()) if failed else torch.equal(a, b), polls
    finally:
        binding.debug_linear_ce_wait_polls(-1)
    after = [c.fwd(binding)] + [[t for t in c.bwd(binding, lse, want=w, dw_f32=f) if t is not None] for w, f in wants]
    for g, ref in zip(after, [fwd] + bwd):
        assert all(torch.equal(a, b) for a, b in zip(g, ref))


@gpu
@pytest.mark.parametrize("shape", [(300, 4096, 700), (70, 2056, 3000)], ids=lambda s: "x".join(map(str, s)))
def test_linear_ce_wide_outputs_asked_for_alone(binding, shape):
    """More than 2048 columns: the logits of the backward pass come out of chains that do not depend on what is asked for."""
    c = Ce(*shape, 1, True, 0.2, seed=61).reference()
    lse = c.lse.float()
    full = c.bwd(binding, lse)
    for got, ref, tol, what in zip(full, (c.dx, c.dw, c.db), (c.e_dx, c.e_dw, c.e_db), ("dx", "dW", "db")):
        within(got, ref, tol, what)
    for k, want in enumerate("xwb"):
        assert torch.equal(c.bwd(binding, lse, want=want)[k], full[k]), want


@gpu
def test_linear_ce_weight_gradient_of_the_most_rows(binding):
    """2^24 rows, all terms of a sum of one sign: W = 0 makes every probability 1 / 128, and x is in [1, 2)."""
    B, D, V = 1 << 24, 8, 128
    g = torch.Generator(device="cuda")
    g.manual_seed(71)
    x = (torch.rand(B, D, device="cuda", generator=g) * 0.99 + 1).to(torch.bfloat16)
    w, labels = torch.zeros(V, D, device="cuda", dtype=torch.bfloat16), torch.zeros(B, device="cuda", dtype=torch.int32)
    lse, dw = f32(B, fill=math.log(V)), torch.full_like(w, 7.0)
    ws = torch.empty(binding.linear_ce_workspace_bytes(1, B, D, V, True), dtype=torch.uint8, device="cuda")
    binding.linear_ce_bwd(1, x, w, None, labels, lse, None, None, None, dw, None, ws, B, D, V)
    mean = x.double().mean(0)
    ref = mean[None, :].expand(V, D) / V
    ref = torch.cat([ref[:1] - mean[None, :], ref[1:]])
    # dz: 2^-20 of the exponential; 1 / 128 and 1 / 128 - 1 are bf16 values.  Chains of 128 steps that lose four units each;
    # 2^24 / 2048 pieces added up one after the other, half a unit each of a sum that grows evenly; the factor, the result
    tol = U[torch.bfloat16] + 2.0 ** -20 + 128 * 4 * 2.0 ** -24 + 8192 / 2 * 2.0 ** -24 + 2.0 ** -23
    within(dw, ref, tol * ref.abs(), "dW")


@gpu
@pytest.mark.parametrize("group,C", [(0, 4096), (128, 4096), (0, 4093), (0, 200)])
def test_add_rmsnorm_8_bit_values_are_the_rounded_quotients(binding, group, C):
    """y8 is y / scale8 rounded to e4m3, value for value: fp32 tensors, whose y and scale8 are what the kernel divides."""
    rows = (1 << 24) // C
    x, res, gamma = rms_inputs(rows, C, 0, 35)
    h, y = torch.empty_like(x), torch.empty_like(x)
    q, scale = torch.empty(rows, C, dtype=torch.float8_e4m3fn, device="cuda"), f32(rows, C // (group or C))
    binding.add_rmsnorm_fwd(0, x, res, gamma, h, y, q, scale, None, rows, C, group)
    want = (y.view(rows, -1, group or C) / scale[..., None]).to(torch.float8_e4m3fn).view(rows, C)
    assert int((want.view(torch.uint8) != q.view(torch.uint8)).sum()) == 0


@gpu
def test_add_rmsnorm_to_8_bits_of_an_infinite_value(binding):
    """y beyond fp32: the scale is infinite, the group's finite values are zero and the infinite one is NaN, as y / scale8 says."""
    rows, C = 3, 256
    x, gamma = torch.ones(rows, C, device="cuda"), torch.ones(C, device="cuda")
    x[1, 7] = 4.0
    gamma[7] = 3e38
    q, scale = torch.empty(rows, C, dtype=torch.float8_e4m3fn, device="cuda"), f32(rows, 2)
    binding.add_rmsnorm_fwd(0, x, None, gamma, None, None, q, scale, None, rows, C, 128)
    assert math.isinf(float(scale[1, 0])) and torch.isfinite(scale[0]).all() and float(scale[1, 1]) > 0
    one = q[1].float()
    assert math.isnan(float(one[7])) and not one[:7].any() and not one[8:128].any() and (one[128:] == 448.0).all()
    assert float(q[0, 7].float()) == 448.0 and float(q[2, 7].float()) == 448.0


@gpu
@PREC
def test_linear_ce_gradients_past_32_bits(binding, prec):
    """dx and the ends of dW of a projection of more than 2^31 values, few rows and many."""
    V, D = 131073 + 64, 16384
    w = torch.empty(V, D, dtype=DT[prec], device="cuda").normal_().mul_(0.01)
    dw = torch.empty_like(w)
    for B in (3, 70):
        c = Ce(B, D, 8, prec, seed=81)
        c.V, c.w = V, w
        c.labels = torch.arange(V - B, V, device="cuda", dtype=torch.int32)
        x = c.x.double()
        parts = torch.cat([x @ w[i: i + 8192].double().t() for i in range(0, V, 8192)], 1)
        ref = torch.logsumexp(parts, 1)
        dx = torch.full_like(c.x, 7.0)
        ws = torch.empty(binding.linear_ce_workspace_bytes(prec, B, D, V, True), dtype=torch.uint8, device="cuda")
        binding.linear_ce_bwd(prec, c.x, w, None, c.labels, ref.float(), None, None, dx, dw, None, ws, B, D, V)
        del ws
        p = (parts - ref[:, None]).exp() / B
        dz = p.clone()
        dz[torch.arange(B), V - B + torch.arange(B)] -= 1.0 / B
        # logits: a step of 16 products loses four units of 2^-24 of sums below 16384 x 0.8 x 0.8 x 0.01 (six products of fp32
        # terms share the sum's 24 bits); exp2 and its argument 2^-20
        tol = 4 * (6 if prec == 0 else 1) * 1024 * 2.0 ** -24 * 110 + 2.0 ** -20
        edz = p * tol + 2.0 ** -24 / B + dz.abs() * (2.0 ** -8 if prec else 2.0 ** -24)
        steps = (4 * (6 if prec == 0 else 1) * math.ceil(V / 16) + 80) * 2.0 ** -24
        want, mass = torch.zeros(B, D, dtype=torch.float64, device="cuda"), torch.zeros(B, D, dtype=torch.float64, device="cuda")
        for i in range(0, V, 8192):
            block = w[i: i + 8192].double()
            want += dz[:, i: i + 8192] @ block
            mass += (edz[:, i: i + 8192] + steps * dz[:, i: i + 8192].abs()) @ block.abs()
        within(dx, want, mass + U[dx.dtype] * want.abs(), "dx")
        for at in (slice(0, 100), slice(V - 100, V)):
            want, mass = dz[:, at].t() @ x, (edz[:, at] + 1100 * 2.0 ** -24 * dz[:, at].abs()).t() @ x.abs()
            within(dw[at], want, mass + U[dw.dtype] * want.abs() + 1e-30, "dW")


@gpu
@PREC
def test_add_rmsnorm_rstd_of_the_widest_rows(binding, prec):
    """16384 columns: a thread adds at most 32 squares (8 per vector, 4 vectors), a tree over 1024 threads 10 more; half of
    that after the root; the sum of x and res, the mean, eps: 2; rsqrt: 4 units of 2^-24."""
    rows, C = 65, 16384
    x, res, gamma = rms_inputs(rows, C, prec, 37)
    h, y, rstd = torch.empty_like(x), torch.empty_like(x), f32(rows)
    binding.add_rmsnorm_fwd(prec, x, res, gamma, h, y, None, None, rstd, rows, C)
    _, ref, y_ref = rms_reference(x, res, gamma, 1e-6)
    e = (42 / 2 + 2 + 4) * 2.0 ** -24
    within(rstd, ref, e * ref, "rstd")
    within(y, y_ref, (U[x.dtype] + e + 3 * 2.0 ** -24) * y_ref.abs(), "y")


def test_philox_of_ones_and_of_the_digits_of_pi():
    """The other published known answers (Salmon et al., 2011); the fourth word of the counter is always zero in a call, so
    the ten rounds are written out for all four words here."""
    def words(c, k):
        for _ in range(10):
            p, q = c[0] * 0xD2511F53, c[2] * 0xCD9E8D57
            c = [(q >> 32) ^ c[1] ^ k[0], q % 2 ** 32, (p >> 32) ^ c[3] ^ k[1], p % 2 ** 32]
            k = [(k[0] + 0x9E3779B9) % 2 ** 32, (k[1] + 0xBB67AE85) % 2 ** 32]
        return c

    one = 2 ** 32 - 1
    assert words([one] * 4, [one] * 2) == [0x408F276D, 0x41C83B0E, 0xA20BC7C6, 0x6D5451FD]
    assert words([0x243F6A88, 0x85A308D3, 0x13198A2E, 0x03707344], [0xA4093822, 0x299F31D0]) == [0xD16CFE09, 0x94FDCCEB, 0x5001E420, 0x24126EA1]
    assert words([0x89ABCDEF, 0x01234567, 7, 0], [0x9ABCDEF0, 0x12345678]) == philox(0x123456789ABCDEF0, 0x0123456789ABCDEF, 7, 1)[0].tolist()


@gpu
@pytest.mark.parametrize("B", [1, 16, 20, 64])
def test_linear_ce_few_rows_cut_their_chains(binding, B):
    """Logits whose 2048 products have one sign: chains of 256, 512 or 1024 products (16, 32, 64 rows at most) whose steps of
    16 lose less than a unit of the sum so far, 2^-23, each, and whose sums are then added rounded to nearest."""
    D, V = 2048, 1000
    g = torch.Generator(device="cuda")
    g.manual_seed(91)
    c = Ce(B, D, 8, 1, seed=92)
    c.x = (torch.rand(B, D, device="cuda", generator=g) + 1).bfloat16()
    c.V, c.w = V, ((torch.rand(V, D, device="cuda", generator=g) + 1) * 2.0 ** -8).bfloat16()
    z = c.x.double() @ c.w.double().t()
    ref = torch.logsumexp(z, 1)
    chain = 256 if B <= 16 else (512 if B <= 32 else 1024)
    # half of the steps' units, as the sum grows; half a unit of 2^-24 for each of the pieces; lse: exp2, the sums in pieces of 128
    # and a tree, the logarithm and its sum
    e = (chain / 16 + 1) / 2 * 2.0 ** -23 + (D / chain + 1) / 2 * 2.0 ** -24
    tol = e * float(z.max()) + 2.0 ** -21 + 100 * 2.0 ** -24 + 8 * 2.0 ** -24 * float(ref.max())
    within(c.fwd(binding)[2], ref, tol, "lse")


@gpu
@pytest.mark.parametrize("shape", [(1, 104, 2277), (2, 136, 3000), (5, 392, 900), (16, 200, 3001), (17, 1000, 2000), (32, 72, 5000)], ids=lambda s: "x".join(map(str, s)))
def test_linear_ce_gradients_of_the_fewest_rows_keep_two_terms_of_dz(binding, shape):
    """Up to 32 rows of bf16: dz enters the products with 16 bits, so that a gradient that a few of its values make up is off
    by its own rounding alone."""
    for ignored in (0.0, 0.3):
        c = Ce(*shape, 1, True, ignored, seed=95).reference(dloss=0.75)
        lse = c.lse.float()
        dx, dw, db = c.bwd(binding, lse, dloss=f32(1, fill=0.75))
        counted = (c.labels >= 0) & (c.labels < c.V)
        y = c.labels.clamp(0, c.V - 1).long()[:, None]
        p = torch.softmax(c.z, 1)
        g = torch.where(counted, 0.75 / max(1, int(counted.sum())), 0.0)[:, None]
        dz = (p - torch.zeros_like(p).scatter_(1, y, 1.0)) * g
        # as in the reference above, with two roundings of 2^-8 of dz one after the other; both terms' products are chains of one
        # step more
        ep = (p * (c.ez + c.e_lse[:, None] + 2.0 ** -21 + 2.0 ** -23 * (c.z - c.lse[:, None]).abs()) + 2.0 ** -24) * g
        edz = ep + 2.0 ** -16 * dz.abs()
        aw, ax, az = c.w.double().abs(), c.x.double().abs(), dz.abs()
        steps = (4 * math.ceil(c.V / 16) + 84) * 2.0 ** -24
        within(dx, c.dx, edz @ aw + steps * (az @ aw) + U[dx.dtype] * c.dx.abs() + 1e-30, "dx")
        within(dw, c.dw, edz.t() @ ax + 40 * 2.0 ** -24 * (az.t() @ ax) + U[dw.dtype] * c.dw.abs() + 1e-30, "dW")
        within(db, c.db, c.e_db, "db")


@gpu
@pytest.mark.parametrize("B,D,V", [(70, 2048, 300), (600, 4096, 1000)])
def test_linear_ce_chains_of_logits_are_short(binding, B, D, V):
    """A product of one and then thousands whose sixteens are a little below the unit of one, 2^-23: what a chain that truncates
    loses altogether.  At most the first 1024 products (64 steps) are one chain with the one; the others add up unharmed."""
    c = Ce(B, D, 8, 1, seed=96)
    c.V = V
    c.x = torch.ones(B, D, device="cuda").bfloat16()
    c.w = torch.full((V, D), 0.8984375 * 2.0 ** -27, device="cuda").bfloat16()
    c.w[:, 0] = 1.0
    c.labels = torch.zeros(B, device="cuda", dtype=torch.int32)
    z = 1.0 + (D - 1) * 0.8984375 * 2.0 ** -27
    loss, row, lse = c.fwd(binding)
    # every exponential is one, their sum exact; the logarithm of V and its sum with z: two units each of values below 8
    tol = 65 * 2.0 ** -23 + 2.0 ** -23 + 4 * 2.0 ** -22
    within(lse, torch.full((B,), math.log(V) + z, dtype=torch.float64, device="cuda"), tol, "lse")

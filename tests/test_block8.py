"""Rows of 8-bit codes, the linear layer on them, and the norms around a block with its gate and residual scale, against
plain implementations in 64 bits.

Tolerances count roundings.  A rounding to a type is off by at most U[type] relative to the value (half a step).  The
tensor cores add 16 products and the accumulator at a time; every such step is taken to lose at most four units of 2^-24
of the sum of the absolute values."""
import math
import os
import subprocess
import sys

import pytest
import torch

from tests.test_lm_ops import DT, INF, NAN, PREC, U, P, Ws, f32, gpu, randn, status, within

E = 2.0 ** -24
ids = lambda s: "x".join(map(str, s))  # noqa: E731


@pytest.fixture
def binding():
    from paper_1804_10574_b200 import binding as b
    return b


# ---- rows of codes --------------------------------------------------------------------------------------------------
LEAST = 127.0 * 2.0 ** -126


def codes(x):
    """Codes, which are whole numbers exactly, and scales of finite rows."""
    top = x.double().abs().amax(1, keepdim=True).clamp(min=LEAST)
    # 127 x is exact in 64 bits, and the quotient of two such values is not near enough to a border to be rounded onto it
    # (a tensor of 127: torch divides by a number on the host by multiplying with its reciprocal)
    return (127 * x.double() / top).round(), (top.float() / torch.full_like(top, 127.0, dtype=torch.float32)).clamp(max=8454659.0 * 2.0 ** 98)[:, 0]


def pack(binding, x, prec, stream=None):
    rows, C = x.shape
    q, scale = torch.full((rows, binding.act8_pitch(C)), 99, dtype=torch.int8, device="cuda"), f32(rows)
    binding.act8_pack(prec, x, q, scale, rows, C, stream)
    return q, scale


def value(q, scale, C, prec):
    """What codes stand for, in the element type."""
    return (q[:, :C].float() * scale[:, None]).to(DT[prec])


ACT_SHAPES = [(1, 1), (1, 16), (3, 7), (5, 64), (130, 128), (2, 1000), (9, 1021), (33, 1024), (4, 4096), (700, 136), (3, 5000), (2, 8192), (3, 16384), (2, 16383), (1, 16385),
              (2, 65536), (1, 131072), (1300, 40), (257, 200), (299, 4096), (400, 8192), (300, 1021), (297, 5000), (310, 2051), (300, 16384)]


@gpu
@PREC
@pytest.mark.parametrize("shape", ACT_SHAPES, ids=ids)
def test_act8_codes_are_the_rounded_quotients(binding, shape, prec):
    """Codes and scales to the last bit, zeros behind a row's codes; unpacking gives their products, rounded once."""
    rows, C = shape
    x = randn(rows, C, seed=3, prec=prec) * torch.logspace(-3, 3, rows, device="cuda").to(DT[prec])[:, None]
    # values on the border of two codes: halves of steps of a row whose maximum is 127 (and of its multiples by powers of two)
    if C >= 64:
        x[0] = (torch.arange(C, device="cuda") % 255 - 127).to(DT[prec]) / 2
        x[0, 5] = 127.0
        x[rows - 1, : C // 2] = x[rows - 1].abs().max() / 2
    q, scale = pack(binding, x, prec)
    ref, s = codes(x)
    assert torch.equal(q[:, :C].double(), ref) and torch.equal(scale, s)
    assert not q[:, C:].any()
    back = torch.full_like(x, 7.0)
    binding.act8_unpack(prec, q, scale, back, rows, C)
    assert torch.equal(back, value(q, scale, C, prec))
    within(back, x, (scale.double()[:, None] / 2) * (1 + 2.0 ** -20) + U[x.dtype] * x.double().abs() * 1.01 + 1e-44, "the row and what its codes stand for")


@gpu
def test_act8_codes_near_borders_of_32_bit_values(binding):
    """Values one unit of fp32 above and below the border of two codes."""
    top = torch.tensor([1.0, 1.9999999, 3.3, 1e-30, 7e30, 0.1], device="cuda")
    k = torch.arange(-127, 127, device="cuda").double() + 0.5
    border = (k[None] * top.double()[:, None] / 127).float()
    x = torch.cat([border, torch.nextafter(border, torch.full_like(border, INF)), torch.nextafter(border, torch.full_like(border, -INF)), top[:, None]], 1)
    q, scale = pack(binding, x, 0)
    ref, s = codes(x)
    assert torch.equal(q[:, : x.shape[1]].double(), ref) and torch.equal(scale, s)


@gpu
@PREC
@pytest.mark.parametrize("C", [40, 4096, 20000])
def test_act8_special_rows(binding, C, prec):
    """Zeros, tiny values, the type's largest; NaN and infinities make their own row NaN and no other."""
    x = randn(8, C, seed=4, prec=prec)
    x[1] = 0.0
    x[2] = randn(C, seed=5, prec=prec) * 2.0 ** -130
    x[3, 7] = torch.finfo(x.dtype).max
    x[4, 9], x[5, 3], x[6, C - 1] = NAN, INF, -INF
    q, scale = pack(binding, x, prec)
    for r in (4, 5, 6):
        assert math.isnan(float(scale[r])) and not q[r].any()
    good = [0, 1, 2, 3, 7]
    ref, s = codes(x[good])
    assert torch.equal(q[good][:, :C].double(), ref) and torch.equal(scale[good], s)
    back = torch.empty_like(x)
    binding.act8_unpack(prec, q, scale, back, 8, C)
    assert torch.isnan(back[4:7]).all() and torch.isfinite(back[good]).all() and not back[1].any()


@gpu
@PREC
def test_act8_off_16_byte_boundaries_and_rows_behind(binding, prec):
    """Tensors that start anywhere; rows behind the last are left as they were."""
    for rows, C in ((33, 256), (20, 77)):
        store = randn(rows * C + 1, seed=6, prec=prec)
        x = store[1:].view(rows, C)
        q, scale = pack(binding, x, prec)
        ref, s = codes(x)
        assert torch.equal(q[:, :C].double(), ref) and torch.equal(scale, s)
        back = torch.full((rows * C + 1,), 7.0, dtype=x.dtype, device="cuda")
        binding.act8_unpack(prec, q, scale, back[1:], rows - 2, C)
        assert torch.equal(back[1:1 + (rows - 2) * C].view(-1, C), value(q, scale, C, prec)[: rows - 2])
        assert float(back[0]) == 7 and (back[1 + (rows - 2) * C:] == 7).all()
        q2, s2 = torch.full_like(q, 5), f32(rows)
        binding.act8_pack(prec, x, q2, s2, rows - 2, C)
        assert (q2[rows - 2:] == 5).all() and (s2[rows - 2:] == 7).all() and torch.equal(q2[: rows - 2], q[: rows - 2])


# ---- the linear layer -----------------------------------------------------------------------------------------------
class Fc:
    """Codes of x and W, dy, the 64-bit reference and its tolerances."""

    def __init__(self, B, D, V, prec, bias=False, seed=0):
        self.B, self.D, self.V, self.prec = B, D, V, prec
        x, w = randn(B, D, seed=seed + 1, prec=prec), randn(V, D, seed=seed + 2, prec=prec, std=1.0 / math.sqrt(D))
        x *= torch.logspace(-1, 1, B, device="cuda").to(x.dtype)[:, None]
        self.bias = randn(V, seed=seed + 3, prec=prec) if bias else None
        self.dy = randn(B, V, seed=seed + 4, prec=prec)
        from paper_1804_10574_b200 import binding as b
        (self.xq, self.xs), (self.wq, self.ws) = pack(b, x, prec), pack(b, w, prec)

    def y_ref(self, u):
        prod = (self.xq[:, : self.D].double() @ self.wq[:, : self.D].double().t()) * self.xs.double()[:, None] * self.ws.double()
        y = prod if self.bias is None else prod + self.bias.double()
        # the sum as a float, two products, the addition
        return y, 4 * E * (prod.abs() + (self.bias.double().abs() if self.bias is not None else 0.0)) + u * y.abs()

    def grads_ref(self, dw_u=None):
        dy, x, w = self.dy.double(), value(self.xq, self.xs, self.D, self.prec).double(), value(self.wq, self.ws, self.D, self.prec).double()
        if self.prec == 0:  # the library may take the product with the scale elsewhere: nothing is rounded there in 64 bits
            x, w = self.xq[:, : self.D].double() * self.xs.double()[:, None], self.wq[:, : self.D].double() * self.ws.double()[:, None]
        parts, u = (3, 4 * E) if self.prec == 0 else (1, 0.0)
        mx, mw = dy.abs() @ w.abs(), dy.abs().t() @ x.abs()
        ex = (4 * parts * math.ceil(self.V / 16) + 16) * E * mx + u * mx
        ew = (4 * parts * math.ceil(self.B / 16) + 16) * E * mw + u * mw
        dx, dw, db = dy @ w, dy.t() @ x, dy.sum(0)
        ut = U[DT[self.prec]]
        return (dx, ex + ut * dx.abs() + 1e-30), (dw, ew + (ut if dw_u is None else dw_u) * dw.abs() + 1e-30), (db, (math.ceil(self.B / 4) + 16) * E * dy.abs().sum(0))  # no chain of additions is longer

    def fwd(self, b, y_f32=False, stream=None, y=None):
        y = torch.full((self.B, self.V), 7.0, dtype=torch.float32 if y_f32 else DT[self.prec], device="cuda") if y is None else y
        b.fc8_fwd(self.prec, self.xq, self.xs, self.wq, self.ws, self.bias, y, self.B, self.D, self.V, y_f32, stream)
        return y

    def bwd(self, b, want="xwb", dw_f32=False, stream=None, ws=None):
        if ws is None:
            ws = torch.full((b.fc8_workspace_bytes(self.prec, self.B, self.D, self.V),), 255, dtype=torch.uint8, device="cuda")
        dx = torch.full((self.B, self.D), 7.0, dtype=DT[self.prec], device="cuda") if "x" in want else None
        dw = torch.full((self.V, self.D), 7.0, dtype=torch.float32 if dw_f32 else DT[self.prec], device="cuda") if "w" in want else None
        db = f32(self.V) if "b" in want else None
        b.fc8_bwd(self.prec, self.dy, self.xq if dw is not None else None, self.xs if dw is not None else None, self.wq if dx is not None else None,
                  self.ws if dx is not None else None, dx, dw, db, ws, self.B, self.D, self.V, dw_f32, stream)
        return dx, dw, db


FC_SHAPES = [(1, 1, 1), (1, 16, 16), (1, 64, 100), (3, 5, 7), (1, 4096, 513), (2, 1000, 4099), (16, 256, 2000), (17, 130, 257), (33, 1000, 1001), (64, 2048, 640), (65, 128, 640),
             (128, 128, 128), (130, 72, 257), (200, 4097, 300), (257, 264, 513), (300, 521, 1000), (511, 16, 255), (700, 2200, 90), (2050, 136, 520), (40, 8200, 33),
             (1100, 300, 2000), (2200, 72, 2300), (2200, 2300, 136), (136, 2300, 2200), (1300, 1408, 3000)]


@gpu
@PREC
@pytest.mark.parametrize("shape", FC_SHAPES, ids=ids)
def test_fc8_forward(binding, shape, prec):
    """One row to several tiles, sizes that fill no tile; with and without a bias; 32-bit results of 16-bit layers."""
    for bias, y_f32 in ((False, False), (True, False), (True, True)):
        c = Fc(*shape, prec, bias, seed=5)
        y, tol = c.y_ref(E if y_f32 else U[DT[prec]])
        within(c.fwd(binding, y_f32), y, tol, "y")


@gpu
@PREC
@pytest.mark.parametrize("shape", FC_SHAPES, ids=ids)
def test_fc8_backward(binding, shape, prec):
    for dw_f32 in (False, True):
        c = Fc(*shape, prec, seed=6)
        refs = c.grads_ref(E if dw_f32 else None)
        for got, (ref, tol), what in zip(c.bwd(binding, dw_f32=dw_f32), refs, ("dx", "dW", "db")):
            within(got, ref, tol, what)


@gpu
@PREC
@pytest.mark.parametrize("shape", [(3000, 300, 200), (200, 300, 3000), (2600, 8200, 2604), (5000, 4100, 2300)], ids=ids)
def test_fc8_gradients_that_share_a_launch(binding, shape, prec):
    """Either product the longer one, their K ranges split or not; so many tiles that each has a launch of its own; both results
    the same bits as alone."""
    for dw_f32 in (False, True):
        c = Fc(*shape, prec, seed=8)
        full = c.bwd(binding, dw_f32=dw_f32)
        for got, (ref, tol), what in zip(full, c.grads_ref(E if dw_f32 else None), ("dx", "dW", "db")):
            within(got, ref, tol, what)
        for k, want in enumerate("xw"):
            assert torch.equal(c.bwd(binding, want, dw_f32)[k], full[k]), want


@gpu
@pytest.mark.parametrize("shape", [(289, 896, 363), (483, 962, 2782), (300, 1024, 4096), (2782, 962, 483), (1400, 520, 340)], ids=ids)
def test_fc8_gradients_whose_chains_are_cut_in_one_product_only(binding, shape):
    """fp32: chains of one product end within the limit, those of the other are cut; the bits are those of each alone."""
    c = Fc(*shape, 0, seed=58)
    full = c.bwd(binding)
    for got, (ref, tol), what in zip(full, c.grads_ref(E), ("dx", "dW", "db")):
        within(got, ref, tol, what)
    for k, want in enumerate("xw"):
        assert torch.equal(c.bwd(binding, want)[k], full[k]), want


@gpu
@PREC
@pytest.mark.parametrize("shape", [(1, 64, 100), (45, 136, 1000), (300, 136, 777), (140, 2000, 90)], ids=ids)
def test_fc8_gradients_asked_for_alone(binding, shape, prec):
    """The same bits whichever are asked for, and again."""
    c = Fc(*shape, prec, seed=7)
    for dw_f32 in (False, True):
        full = c.bwd(binding, dw_f32=dw_f32)
        for k, want in enumerate("xwb"):
            assert torch.equal(c.bwd(binding, want, dw_f32)[k], full[k]), want
        for k, want in ((0, "xb"), (1, "wb"), (2, "wb"), (0, "xw")):
            assert torch.equal(c.bwd(binding, want, dw_f32)[k], full[k]), want


@gpu
@PREC
@pytest.mark.parametrize("shape", [(1, 4096, 200), (20, 4096, 200), (300, 16384, 64), (2, 131072, 40), (300, 131072, 70)], ids=ids)
def test_fc8_largest_sums(binding, shape, prec):
    """All codes 127 or -127: the largest sums that a row can have, exact in 32 bits."""
    B, D, V = shape
    c = Fc(*shape, prec, seed=8)
    c.xq[:, :D] = 127
    c.wq[:, :D] = 127
    c.wq[V // 2:, :D] = -127
    c.xs.fill_(2.0 ** -7)
    c.ws.fill_(2.0 ** -9)
    y = c.fwd(binding, True)
    ref = torch.full((V,), 127.0 * 127.0 * D * 2.0 ** -16, dtype=torch.float64, device="cuda")
    ref[V // 2:] *= -1
    assert torch.equal(y, ref.float().expand(B, V))  # rounded once: the scales are powers of two


@gpu
@PREC
@pytest.mark.parametrize("shape", [(3, 4096, 100), (300, 2048, 260), (40, 1000, 33)], ids=ids)
def test_fc8_scales_of_unlike_size(binding, shape, prec):
    """Rows of x near the type's largest values and small weights, and the other way round: the products are of ordinary size."""
    for s, bias in ((2.0 ** 117, False), (2.0 ** -117, True), (2.0 ** 90, True)):
        c = Fc(*shape, prec, bias, seed=60)
        c.xq[0, : c.D] = 127
        c.wq[:2, : c.D] = 127
        c.xs *= s
        c.ws /= s
        y, tol = c.y_ref(U[DT[prec]])
        within(c.fwd(binding), y, tol, "y")


@gpu
@PREC
def test_fc8_does_not_read_behind_a_rows_codes(binding, prec):
    """Whatever stands in the bytes that fill a row up."""
    for shape in ((1, 1001, 300), (40, 71, 130), (300, 521, 270)):
        c = Fc(*shape, prec, seed=9)
        ref = [c.fwd(binding)] + list(c.bwd(binding))
        c.xq[:, c.D:], c.wq[:, c.D:] = 77, -99
        for a, b in zip(ref, [c.fwd(binding)] + list(c.bwd(binding))):
            assert torch.equal(a, b)


@gpu
@PREC
@pytest.mark.parametrize("shape", [(5, 64, 300), (300, 64, 700)], ids=ids)
def test_fc8_rows_that_are_not_numbers(binding, shape, prec):
    """A row of codes with scale NaN makes its row of y NaN and no other; in dW, where all rows are summed, it shows; dx does
    not see it.  Infinite dy stays in its row of dx."""
    c = Fc(*shape, prec, seed=10)
    clean, clean_dx = c.fwd(binding), c.bwd(binding, "x")[0]
    c.xs[3] = NAN
    y = c.fwd(binding)
    keep = torch.arange(c.B, device="cuda") != 3
    assert torch.isnan(y[3]).all() and torch.equal(y[keep], clean[keep])
    dx, dw, db = c.bwd(binding)
    assert torch.equal(dx, clean_dx) and torch.isnan(dw).all() and torch.isfinite(db).all()
    c.dy[2, 5] = INF
    dx = c.bwd(binding, "x")[0]
    keep = torch.arange(c.B, device="cuda") != 2
    assert torch.equal(dx[keep], clean_dx[keep]) and not torch.isfinite(dx[2].float()).any()
    c.ws[7] = NAN
    y = c.fwd(binding)
    assert torch.isnan(y[:, 7]).all() and torch.isfinite(y[keep & (torch.arange(c.B, device="cuda") != 3)][:, :7]).all()


@gpu
def test_fc8_gradient_of_products_past_the_largest_bf16(binding):
    """fp32: dy times the scale may be up to the largest fp32 value, which is past bf16's; it has to reach neither its columns of
    codes 0 nor, as an infinity, the others."""
    B, D, V = 300, 72, 200
    c = Fc(B, D, V, 0, seed=61)
    c.dy.zero_()
    big = 3.3999e38
    c.dy[5, 9], c.dy[7, 150] = big, -big
    c.ws.fill_(1.0)
    c.xs.fill_(1.0)
    for q in (c.wq, c.xq):
        q[:, :D] = (torch.arange(D, device="cuda") % 3 - 1).to(torch.int8)
    dx, dw, _ = c.bwd(binding, "xw")
    e = torch.zeros(B, D, dtype=torch.float64, device="cuda")
    e[5], e[7] = big * c.wq[9, :D].double(), -big * c.wq[150, :D].double()
    within(dx, e, 16 * E * e.abs(), "dx")
    e = torch.zeros(V, D, dtype=torch.float64, device="cuda")
    e[9], e[150] = big * c.xq[5, :D].double(), -big * c.xq[7, :D].double()
    within(dw, e, 16 * E * e.abs(), "dW")


@gpu
def test_fc8_gradient_against_differences(binding):
    """The layer is linear in what the codes stand for: steps of whole codes change <dy, y> by the gradients' products."""
    c = Fc(37, 200, 150, 0, seed=11)
    dx, dw, _ = c.bwd(binding)
    base = (c.fwd(binding).double() * c.dy.double()).sum()
    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    for q, s, grad in ((c.xq, c.xs, dx), (c.wq, c.ws, dw)):
        step = torch.randint(-1, 2, q.shape, device="cuda", generator=g, dtype=torch.int8)
        step[:, c.D:] = 0
        step[(q.int() + step).abs() > 127] = 0
        kept = q.clone()
        q += step
        moved = (c.fwd(binding).double() * c.dy.double()).sum() - base
        q.copy_(kept)
        said = (grad.double() * (step[:, : c.D].double() * s.double()[:, None])).sum()
        y, tol = c.y_ref(E)
        # each of the two sums: y's error; the gradient's own error is counted in roundings of the same products
        allowed = 4 * (tol * c.dy.double().abs()).sum() + 100 * E * (grad.double().abs() * step[:, : c.D].double().abs() * s.double()[:, None]).sum()
        assert abs(float(moved - said)) <= float(allowed)


@gpu
@PREC
def test_fc8_off_16_byte_boundaries(binding, prec):
    """y, dy, bias and the gradients may start anywhere; odd widths."""
    for shape in ((5, 64, 300), (300, 65, 700), (130, 264, 513), (1, 333, 77)):
        c = Fc(*shape, prec, True, seed=12)
        ref_y, ref = c.fwd(binding), c.bwd(binding)
        e = DT[prec]
        store = [torch.full((n + 1,), 7.0, dtype=t, device="cuda") for n, t in ((c.B * c.V, e), (c.B * c.D, e), (c.V * c.D, e))]
        dy, bias = torch.empty(c.B * c.V + 1, dtype=e, device="cuda"), torch.empty(c.V + 1, dtype=e, device="cuda")
        dy[1:], bias[1:] = c.dy.flatten(), c.bias
        y, dx, dw = (t[1:] for t in store)
        binding.fc8_fwd(prec, c.xq, c.xs, c.wq, c.ws, bias[1:], y, *shape)
        ws = torch.full((binding.fc8_workspace_bytes(prec, *shape) + 256,), 77, dtype=torch.uint8, device="cuda")
        binding.fc8_bwd(prec, dy[1:], c.xq, c.xs, c.wq, c.ws, dx, dw, None, ws[:-256], *shape)
        assert torch.equal(y.view_as(ref_y), ref_y)
        refs = c.grads_ref()
        within(dx.view_as(ref[0]), *refs[0], "dx")
        within(dw.view_as(ref[1]), *refs[1], "dW")
        assert all(float(t[0]) == 7 for t in store) and (ws[-256:] == 77).all()


@gpu
@PREC
@pytest.mark.parametrize("shape", [(1, 1000, 500), (20, 264, 1000), (300, 72, 900)], ids=ids)
def test_fc8_other_stream_and_recorded(binding, shape, prec):
    """On a stream of its own; recorded, and replayed on other inputs in the same buffers; two recorded calls that share a
    workspace; the same bits every time."""
    c, other = Fc(*shape, prec, True, seed=15), Fc(*shape, prec, True, seed=16)
    refs = [[k.fwd(binding)] + list(k.bwd(binding)) for k in (c, other)]
    stream = torch.cuda.Stream()
    ws = torch.empty(binding.fc8_workspace_bytes(prec, *shape), dtype=torch.uint8, device="cuda")
    out = [torch.empty_like(t) for t in refs[0]]
    torch.cuda.synchronize()

    def forward():
        binding.fc8_fwd(prec, c.xq, c.xs, c.wq, c.ws, c.bias, out[0], *shape, False, stream.cuda_stream)

    def backward():
        binding.fc8_bwd(prec, c.dy, c.xq, c.xs, c.wq, c.ws, out[1], out[2], out[3], ws, *shape, False, stream.cuda_stream)

    forward(), backward()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(out, refs[0]))
    graphs = []
    for what in ((forward, backward), (backward,)):
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1], stream=stream):
            for w in what:
                w()
    names = ("xq", "xs", "wq", "ws", "bias", "dy")
    first = [getattr(c, n).clone() for n in names]
    for k in (1, 0, 1):
        for n, t in zip(names, [getattr(other, m) for m in names] if k else first):
            getattr(c, n).copy_(t)
        for o in out:
            o.fill_(3.0)
        torch.cuda.synchronize()
        for g in graphs:
            g.replay()
            torch.cuda.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(out, refs[k])), k


@gpu
def test_fc8_two_streams_at_once(binding):
    pairs = [Fc(300, 72, 4000, 1, True, seed=31), Fc(1, 4096, 9000, 1, True, seed=32), Fc(100, 72, 2000, 0, seed=33), Fc(20, 2048, 3000, 1, seed=34)]
    alone = [[c.fwd(binding)] + list(c.bwd(binding)) for c in pairs]
    streams = [torch.cuda.Stream() for _ in pairs]
    torch.cuda.synchronize()
    for _ in range(3):
        together = []
        for c, s in zip(pairs, streams):
            with torch.cuda.stream(s):
                together.append([c.fwd(binding, stream=s.cuda_stream)] + list(c.bwd(binding, stream=s.cuda_stream)))
        torch.cuda.synchronize()
        for a, t in zip(alone, together):
            assert all(torch.equal(p, q) for p, q in zip(a, t))


@gpu
@PREC
def test_fc8_leaves_what_it_does_not_own(binding, prec):
    """Buffers with more rows than the call names keep the rows behind the last; inputs are not written."""
    for B, V, n, v in ((300, 270, 290, 260), (30, 270, 20, 251), (3, 270, 1, 259)):
        c = Fc(B, 65, V, prec, True, seed=17)
        names = ("xq", "xs", "wq", "ws", "bias", "dy")
        kept = [getattr(c, k).clone() for k in names]
        y, dx, dw, db = torch.full((B * V,), 7.0, dtype=DT[prec], device="cuda"), torch.full((B, 65), 7.0, dtype=DT[prec], device="cuda"), f32(V, 65), f32(V)
        binding.fc8_fwd(prec, c.xq, c.xs, c.wq, c.ws, c.bias, y, n, 65, v)
        ws = torch.empty(binding.fc8_workspace_bytes(prec, n, 65, v), dtype=torch.uint8, device="cuda")
        binding.fc8_bwd(prec, c.dy.flatten(), c.xq, c.xs, c.wq, c.ws, dx, dw, db, ws, n, 65, v, True)
        assert (y[n * v:] == 7).all() and (dx[n:] == 7).all() and (dw[v:] == 7).all() and (db[v:] == 7).all()
        assert torch.isfinite(y.float()).all() and all(torch.equal(a, getattr(c, k)) for a, k in zip(kept, names))


@gpu
def test_block8_refuses_on_the_gpu(binding):
    c = Fc(4, 64, 100, 1, True, seed=18)
    y, ws = c.fwd(binding), torch.empty(binding.fc8_workspace_bytes(1, 4, 64, 100) + 512, dtype=torch.uint8, device="cuda")

    def fwd(xq=c.xq, xs=c.xs, wq=c.wq, bias=c.bias, y=y):
        binding.fc8_fwd(1, xq, xs, wq, c.ws, bias, y, 4, 64, 100)

    def bwd(dy=c.dy, ws=ws, dx=torch.empty(4, 64, dtype=torch.bfloat16, device="cuda"), dw=None):
        binding.fc8_bwd(1, dy, c.xq, c.xs, c.wq, c.ws, dx, dw, None, ws, 4, 64, 100)

    fwd(), bwd()
    need = ws.numel() - 512
    for fn, kw in ((fwd, {"xq": c.xq.data_ptr() + 8}), (fwd, {"xq": c.xq.cpu()}), (fwd, {"y": y.cpu()}), (bwd, {"ws": ws[:need - 1]}), (bwd, {"ws": ws[8:]}), (bwd, {"dy": c.dy.cpu()})):
        with pytest.raises(binding.DdgError) as e:
            fn(**kw)
        assert e.value.status == 1, kw
    for fn, kw in ((fwd, {"xq": c.xq.float()}), (fwd, {"xq": c.xq[:3]}), (fwd, {"xs": c.xs.bfloat16()}), (fwd, {"wq": c.wq.t()}), (fwd, {"y": y.float()}), (fwd, {"bias": c.bias.float()}),
                   (bwd, {"dy": c.dy.float()}), (bwd, {"dx": y[:, :64]}), (bwd, {"dw": torch.empty(100, 64, device="cuda")})):
        with pytest.raises(ValueError):
            fn(**kw)
    torch.cuda.synchronize()


# ---- norms around a block -------------------------------------------------------------------------------------------
EPS, ALPHA = 1e-6, 0.875
# roundings of a mean of squares (32 values per thread and a tree of 10 steps, halved by the root), its division, addition and root
RSTD_E = 27 * E


class Norm:
    def __init__(self, rows, C, prec, span=None, gate=True, seed=0):
        self.rows, self.C, self.prec, self.span = rows, C, prec, span or rows
        self.b, self.res = randn(rows, C, seed=seed + 1, prec=prec), randn(rows, C, seed=seed + 2, prec=prec, std=3.0)
        self.gate = randn(-(-rows // self.span), C, seed=seed + 3, prec=prec, std=0.3, mean=0.5) if gate else None
        self.post, self.pre = randn(C, seed=seed + 4, prec=prec, std=0.2, mean=1.0), randn(C, seed=seed + 5, prec=prec, std=0.2, mean=1.0)
        self.dy, self.dh = randn(rows, C, seed=seed + 6, prec=prec), randn(rows, C, seed=seed + 7, prec=prec)

    def per_row(self):
        g = torch.ones(1, self.C, dtype=torch.float64, device="cuda").expand(self.rows, -1) if self.gate is None else self.gate.double().repeat_interleave(self.span, 0)[: self.rows]
        return g

    def reference(self):
        b, g, post, pre, res = self.b.double(), self.per_row(), self.post.double(), self.pre.double(), self.res.double()
        self.r1 = 1.0 / (b.square().mean(1, keepdim=True) + EPS).sqrt()
        gu = g * b * self.r1 * post
        self.h = ALPHA * res + gu
        self.e_h = (RSTD_E + 4 * E) * gu.abs() + 2 * E * (ALPHA * res).abs() + 1e-44
        ms = self.h.square().mean(1, keepdim=True) + EPS
        self.r2 = 1.0 / ms.sqrt()
        self.e_r2 = RSTD_E + (self.h.abs() * self.e_h).mean(1, keepdim=True) / ms  # relative
        self.y = self.h * self.r2 * pre
        self.e_y = self.r2 * pre.abs() * self.e_h + self.y.abs() * (self.e_r2 + 3 * E) + 1e-44
        return self

    def fwd(self, b, to_y=True, to_q=False, stream=None, h=None, y=None):
        n, C = self.rows, self.C
        h = torch.full_like(self.b, 7.0) if h is None else h
        y = (torch.full_like(self.b, 7.0) if y is None else y) if to_y else None
        q, s = (torch.full((n, b.act8_pitch(C)), 99, dtype=torch.int8, device="cuda"), f32(n)) if to_q else (None, None)
        r1, r2 = f32(n), f32(n)
        b.block_norm_fwd(self.prec, self.b, self.res, self.gate, self.post, self.pre, h, y, q, s, r1, r2, n, C, self.span, ALPHA, EPS, stream)
        return h, y, q, s, r1, r2

    def bwd(self, b, h, r1, r2, dh=True, dgate=True, db=None, dres=None, stream=None):
        n, C = self.rows, self.C
        db, dres = torch.full_like(self.b, 7.0) if db is None else db, torch.full_like(self.b, 7.0) if dres is None else dres
        dg = f32(*self.gate.shape) if self.gate is not None and dgate else None
        dpost, dpre, scratch = f32(C), f32(C), f32(b.block_norm_scratch_elems(n, C, self.span), fill=NAN)
        b.block_norm_bwd(self.prec, self.dy, self.dh if dh else None, self.b, h, self.gate, self.post, self.pre, r1, r2, db, dres, dg, dpost, dpre, scratch, n, C, self.span,
                         ALPHA, stream)
        return db, dres, dg, dpost, dpre

    def grads_ref(self, h, r1, r2, dh=True):
        b, k, g, post, pre, dy = self.b.double(), h.double(), self.per_row(), self.post.double(), self.pre.double(), self.dy.double()
        s1, s2 = r1.double()[:, None], r2.double()[:, None]
        add = self.dh.double() if dh else torch.zeros_like(b)
        # 32 products per thread and a tree of 10 steps, twelve more roundings
        e = 54 * E
        t = add + s2 * (pre * dy - k * s2 * s2 * (pre * dy * k).mean(1, keepdim=True))
        mt = add.abs() + s2 * (pre * dy).abs() + k.abs() * s2 ** 3 * (pre * dy * k).abs().mean(1, keepdim=True)
        w = post * g
        db = s1 * (w * t - b * s1 * s1 * (w * t * b).mean(1, keepdim=True))
        mb = s1 * (w.abs() * mt + b.abs() * s1 * s1 * (w.abs() * mt * b.abs()).mean(1, keepdim=True))
        u = U[self.b.dtype]
        adds = (self.rows + 60) * E  # no chain of additions is longer
        gates = torch.arange(self.rows, device="cuda") // self.span
        n_gates = -(-self.rows // self.span)
        fold = lambda v: torch.zeros(n_gates, self.C, dtype=torch.float64, device="cuda").index_add_(0, gates, v)  # noqa: E731
        unit = b * s1
        return ((db, 2 * e * mb + u * db.abs() + 1e-44), (ALPHA * t, e * ALPHA * mt + u * (ALPHA * t).abs() + 1e-44),
                (fold(t * unit * post), (e + adds) * fold((mt * unit * post).abs()) + 1e-44), ((g * t * unit).sum(0), (e + adds) * (g * mt * unit).abs().sum(0) + 1e-44),
                ((dy * k * s2).sum(0), (4 * E + adds) * (dy * k * s2).abs().sum(0) + 1e-44))


# rows, width, rows per gate
NORM_SHAPES = [(1, 1, 1), (1, 8, 1), (3, 7, 2), (5, 64, 5), (7, 128, 1), (2, 1000, 2), (9, 1021, 3), (33, 1024, 10), (130, 2048, 130), (4, 4096, 1), (700, 136, 100),
               (3, 5000, 3), (2, 8192, 1), (3, 16384, 2), (2, 16383, 1), (1300, 40, 1300), (1300, 40, 1), (900, 520, 7), (350, 4096, 350), (601, 1536, 300), (64, 77, 1),
               (2500, 256, 2500), (2500, 256, 13)]


@gpu
@PREC
@pytest.mark.parametrize("shape", NORM_SHAPES, ids=ids)
def test_block_norm_forward(binding, shape, prec):
    """One row to many, all widths; a gate per row, per sample, for all, none; to the element type, to codes and to both."""
    for gate in (True, False):
        c = Norm(*shape[:2], prec, shape[2], gate, seed=21).reference()
        h, y, q, s, r1, r2 = c.fwd(binding, True, True)
        u = U[h.dtype]
        within(h, c.h, c.e_h + u * c.h.abs(), "h")
        within(r1, c.r1[:, 0], RSTD_E * c.r1[:, 0], "rstd_post")
        within(r2, c.r2[:, 0], (c.e_r2 * c.r2)[:, 0], "rstd_pre")
        within(y, c.y, c.e_y + u * c.y.abs(), "y")
        top = c.y.abs().amax(1).clamp(min=LEAST)
        e_top = c.e_y.amax(1)
        within(s, top / 127, (e_top + 2 * E * top) / 127, "scale")
        got = q[:, : c.C].double() * s.double()[:, None]
        within(got, c.y, s.double()[:, None] * (0.5 + 2.0 ** -12) + 2 * c.e_y.amax(1, keepdim=True), "codes")
        assert not q[:, c.C:].any() and (q.abs().amax(1) == 127).all()
        for to_y, to_q in ((True, False), (False, True)):
            h2, y2, q2, s2, _, _ = c.fwd(binding, to_y, to_q)
            assert torch.equal(h2, h) and (not to_y or torch.equal(y2, y)) and (not to_q or (torch.equal(q2, q) and torch.equal(s2, s)))


@gpu
@PREC
@pytest.mark.parametrize("shape", NORM_SHAPES, ids=ids)
def test_block_norm_backward(binding, shape, prec):
    for gate, dh in ((True, True), (False, True), (True, False)):
        c = Norm(*shape[:2], prec, shape[2], gate, seed=22).reference()
        h, r1, r2 = c.h.to(DT[prec]), c.r1[:, 0].float(), c.r2[:, 0].float()
        got, refs = c.bwd(binding, h, r1, r2, dh), c.grads_ref(h, r1, r2, dh)
        for g, (ref, tol), what in zip(got, refs, ("db", "dres", "dgate", "dgamma_post", "dgamma_pre")):
            if g is not None:
                within(g, ref, tol, what)
        again = c.bwd(binding, h, r1, r2, dh, dgate=False)
        assert all(torch.equal(a, b) for k, (a, b) in enumerate(zip(got, again)) if k != 2)


@gpu
@PREC
@pytest.mark.parametrize("C", [64, 1021, 4096])
def test_block_norm_in_place(binding, C, prec):
    """h and y over b and res; db and dres over what the backward pass reads."""
    c = Norm(20, C, prec, 7, seed=23).reference()
    h, y, _, _, r1, r2 = c.fwd(binding)
    for a, b in (("b", "res"), ("res", "b")):
        k = Norm(20, C, prec, 7, seed=23)
        h2, y2, _, _, _, _ = k.fwd(binding, h=getattr(k, a), y=getattr(k, b))
        assert torch.equal(h2, h) and torch.equal(y2, y)
    ref = c.bwd(binding, h, r1, r2)
    for a, b in (("dy", "dh"), ("dh", "b"), ("b", "dy"), ("h", "dh"), ("b", "h")):
        k = Norm(20, C, prec, 7, seed=23)
        k.h = h.clone()
        got = k.bwd(binding, k.h, r1, r2, db=getattr(k, a), dres=getattr(k, b))
        assert all(torch.equal(p, q) for p, q in zip(got, ref)), (a, b)


@gpu
@PREC
def test_block_norm_special_rows(binding, prec):
    """Rows of zeros, NaN and infinities are their own, also in the codes; a gate of zeros leaves the residual."""
    c = Norm(6, 264, prec, 1, seed=24)
    c.b[1], c.res[1] = 0.0, 0.0
    c.b[2, 7], c.res[3, 9] = NAN, INF
    c.gate[4] = 0.0
    h, y, q, s, r1, r2 = c.fwd(binding, True, True)
    assert not h[1].any() and not y[1].any() and not q[1].any() and float(s[1]) == 2.0 ** -126
    for r in (2, 3):
        assert math.isnan(float(s[r])) and not q[r].any()
    assert torch.isnan(y[2]).all()
    assert torch.equal(h[4], (ALPHA * c.res[4].float()).to(h.dtype))
    for r in (0, 4, 5):
        assert torch.isfinite(y[r].float()).all() and math.isfinite(float(s[r]))


@gpu
@PREC
def test_block_norm_off_16_byte_boundaries(binding, prec):
    for C in (256, 77):
        c = Norm(30, C, prec, 10, seed=25).reference()
        for name in ("b", "res", "gate", "post", "pre", "dy", "dh"):
            t = getattr(c, name)
            store = torch.empty(t.numel() + 1, dtype=t.dtype, device="cuda")
            store[1:] = t.flatten()
            setattr(c, name, store[1:].view(t.shape))
        h, y, q, s, r1, r2 = c.fwd(binding, True, True)
        within(h, c.h, c.e_h + U[h.dtype] * c.h.abs(), "h")
        within(y, c.y, c.e_y + U[h.dtype] * c.y.abs(), "y")
        got, refs = c.bwd(binding, h, r1, r2), c.grads_ref(h, r1, r2)
        for g, (ref, tol), what in zip(got, refs, ("db", "dres", "dgate", "dgamma_post", "dgamma_pre")):
            within(g, ref, tol, what)


@gpu
def test_block_norm_gradient_against_differences(binding):
    """<dy, y> + <dh, h> along a direction of every input, in 32 bits, by central differences in the library's forward pass."""
    c = Norm(24, 520, 0, 8, seed=26)
    h, _, _, _, r1, r2 = c.fwd(binding)
    db, dres, dgate, dpost, dpre = c.bwd(binding, h, r1, r2)
    total = lambda: sum((a.double() * b.double()).sum() for a, b in zip(c.fwd(binding)[:2], (c.dh, c.dy)))  # noqa: E731
    mass = sum((a.double() * b.double()).abs().sum() for a, b in zip(c.fwd(binding)[:2], (c.dh, c.dy)))
    for name, grad in (("b", db), ("res", dres), ("gate", dgate), ("post", dpost), ("pre", dpre)):
        t = getattr(c, name)
        kept, d = t.clone(), randn(*t.shape, seed=77, prec=0)
        got = []
        for step in (2.0 ** -7, -(2.0 ** -7)):
            t.copy_(kept + step * d)
            got.append(float(total()))
        t.copy_(kept)
        slope, said = (got[0] - got[1]) / 2.0 ** -6, float((grad.double() * d.double()).sum())
        # each value of the forward pass is within 60 roundings; the third derivative is bounded by a few times the values'
        # size over a direction of their own size, times step^2 / 6
        allowed = 2 * 60 * E * float(mass) / 2.0 ** -6 + 2.0 ** -14 * float(mass)
        assert abs(slope - said) <= allowed, name


@gpu
@PREC
def test_block_norm_recorded_and_at_once(binding, prec):
    """Recorded and replayed on other inputs; two streams at once; the same bits."""
    a, b = Norm(500, 520, prec, 100, seed=27), Norm(500, 520, prec, 100, seed=28)
    def step(c, stream=None):
        h, y, q, s, r1, r2 = c.fwd(binding, True, True, stream)
        return (h, y, q, s) + c.bwd(binding, h, r1, r2, stream=stream)
    refs = [step(a), step(b)]
    s1, s2 = torch.cuda.Stream(), torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(s1):
        x = step(a, s1.cuda_stream)
    with torch.cuda.stream(s2):
        y = step(b, s2.cuda_stream)
    torch.cuda.synchronize()
    assert all(torch.equal(p, q) for p, q in zip(x, refs[0])) and all(torch.equal(p, q) for p, q in zip(y, refs[1]))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s1):
        out = step(a, s1.cuda_stream)
    for name in ("b", "res", "gate", "post", "pre", "dy", "dh"):
        getattr(a, name).copy_(getattr(b, name))
    for _ in range(2):
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(p, q) for p, q in zip(out, refs[1]))


@gpu
def test_block_norm_more_gates_than_a_grid_has_rows(binding):
    """65600 rows of the gate, each gate's rows worked in two stretches (so many gates are almost a whole number of rounds of the
    resident blocks, so that halves end sooner), in place: the rows repeat after ten gates, so that the results do too."""
    C, span, times = 65, 90, 6560
    c = Norm(10 * span, C, 1, span, seed=57).reference()
    h, r1, r2 = c.h.to(torch.bfloat16), c.r1[:, 0].float(), c.r2[:, 0].float()
    refs = c.grads_ref(h, r1, r2)
    rows = c.rows * times
    dy, dh, b, h, gate = (t.repeat(times, 1) for t in (c.dy, c.dh, c.b, h, c.gate))
    r1, r2 = r1.repeat(times), r2.repeat(times)
    dg, dpost, dpre, scratch = f32(10 * times, C), f32(C), f32(C), f32(binding.block_norm_scratch_elems(rows, C, span), fill=NAN)
    binding.block_norm_bwd(1, dy, dh, b, h, gate, c.post, c.pre, r1, r2, dh, dy, dg, dpost, dpre, scratch, rows, C, span, ALPHA)
    for got, (ref, tol), what in zip((dh, dy, dg), refs, ("db", "dres", "dgate")):
        for k in (0, 1, times // 2, times - 2, times - 1):
            n = ref.shape[0]
            within(got[k * n:(k + 1) * n], ref, tol, what)
        assert torch.equal(got.view(times, -1), got[: ref.shape[0]].reshape(1, -1).expand(times, -1)), what
    for got, (ref, tol), what in zip((dpost, dpre), refs[3:], ("dgamma_post", "dgamma_pre")):
        # chains of additions: of the rows of a block (all SMs have one at least), of the blocks' sums
        mass = tol / ((c.rows + 64) * E)
        within(got, times * ref, (rows / 148 + 2 * span + 2048 + 54) * E * times * mass, what)


@gpu
@PREC
@pytest.mark.parametrize("rows,C", [(20, 264), (700, 1021), (900, 4096)])
def test_block_norm_without_a_gate_does_not_depend_on_span(binding, rows, C, prec):
    got = []
    for span in (rows, 1, 7, 2 * rows):
        c = Norm(rows, C, prec, span, False, seed=59).reference()
        h, r1, r2 = c.h.to(DT[prec]), c.r1[:, 0].float(), c.r2[:, 0].float()
        got.append(c.fwd(binding, True, True)[:4] + tuple(t for t in c.bwd(binding, h, r1, r2) if t is not None))
    for other in got[1:]:
        assert all(torch.equal(a, b) for a, b in zip(got[0], other))


# ---- together -------------------------------------------------------------------------------------------------------
@gpu
@pytest.mark.parametrize("prec,rows,D,F,span", [(1, 300, 264, 520, 100), (0, 130, 72, 257, 130), (1, 24, 1024, 4096, 1)])
def test_block_with_a_history_of_codes(binding, prec, rows, D, F, span):
    """Two steps of a block (norms to codes, linear layer on them) whose backward passes run a step late, from the codes that
    were kept: y = W codes(norm(alpha res + gate norm(b))), the gradients against those of a torch graph with the codes'
    rounding taken as the identity."""
    e = DT[prec]
    w = randn(F, D, seed=61, prec=prec, std=1.0 / math.sqrt(D))
    wq, ws_ = pack(binding, w, prec)
    history, outs = [], []
    for step in range(2):
        c = Norm(rows, D, prec, span, seed=70 + 10 * step)
        h, _, q, s, r1, r2 = c.fwd(binding, False, True)
        y = torch.empty(rows, F, dtype=e, device="cuda")
        binding.fc8_fwd(prec, q, s, wq, ws_, None, y, rows, D, F)
        history.append((c, h, q, s, r1, r2))  # codes instead of the layer's input
        outs.append(y)
    for step, (c, h, q, s, r1, r2) in enumerate(history):
        dy = randn(rows, F, seed=90 + step, prec=prec)
        dn, dw, db = torch.empty(rows, D, dtype=e, device="cuda"), f32(F, D), f32(F)
        work = torch.empty(binding.fc8_workspace_bytes(prec, rows, D, F), dtype=torch.uint8, device="cuda")
        binding.fc8_bwd(prec, dy, q, s, wq, ws_, dn, dw, db, work, rows, D, F, True)
        c.dy = dn
        got = c.bwd(binding, h, r1, r2)
        # the graph in 64 bits
        leaf = {k: getattr(c, k).double().requires_grad_() for k in ("b", "res", "gate", "post", "pre")}
        wl = value(wq, ws_, D, prec).double().requires_grad_()
        g = leaf["gate"].repeat_interleave(span, 0)[:rows]
        hh = ALPHA * leaf["res"] + g * leaf["b"] / (leaf["b"].square().mean(1, keepdim=True) + EPS).sqrt() * leaf["post"]
        nn = hh / (hh.square().mean(1, keepdim=True) + EPS).sqrt() * leaf["pre"]
        kept = nn + (value(q, s, D, prec).double() - nn).detach()
        out = kept @ wl.t()
        (out * dy.double()).sum().add((hh * c.dh.double()).sum()).backward()
        # y: roundings of y and of x^; h and dn are stored rounded, and enter the norms' gradients
        u = 2 * U[e] if prec else 2.0 ** -20
        assert float((outs[step].double() - out.detach()).norm() / out.detach().norm()) < u
        assert float((dw.double() - wl.grad).norm() / wl.grad.norm()) < u
        for a, k in zip(got, ("b", "res", "gate", "post", "pre")):
            assert float((a.double() - leaf[k].grad).norm() / leaf[k].grad.norm()) < 4 * u, k


FIRST_CALL_IS_RECORDED = """
import torch
from paper_1804_10574_b200 import binding as b
n, d, f = 200, 72, 300
bb, res = torch.randn(n, d, device="cuda").bfloat16(), torch.randn(n, d, device="cuda").bfloat16()
one, w, dy = torch.ones(d, device="cuda").bfloat16(), torch.randn(f, d, device="cuda").bfloat16(), torch.randn(n, f, device="cuda").bfloat16()
h, y, dx, dw = torch.empty_like(bb), torch.empty(n, f, device="cuda").bfloat16(), torch.empty_like(bb), torch.empty_like(w)
q, wq = (torch.empty(k, b.act8_pitch(d), dtype=torch.int8, device="cuda") for k in (n, f))
s, ws, r1, r2 = (torch.empty(k, device="cuda") for k in (n, f, n, n))
db, dres, dp, dq = torch.empty_like(bb), torch.empty_like(bb), torch.empty(d, device="cuda"), torch.empty(d, device="cuda")
work, scratch = torch.empty(b.fc8_workspace_bytes(1, n, d, f), dtype=torch.uint8, device="cuda"), torch.empty(b.block_norm_scratch_elems(n, d, n), device="cuda")
stream = torch.cuda.Stream()
def step(st):
    b.act8_pack(1, w, wq, ws, f, d, st)
    b.block_norm_fwd(1, bb, res, None, one, one, h, None, q, s, r1, r2, n, d, n, 1.0, 1e-6, st)
    b.fc8_fwd(1, q, s, wq, ws, None, y, n, d, f, False, st)
    b.fc8_bwd(1, dy, q, s, wq, ws, dx, dw, None, work, n, d, f, False, st)
    b.block_norm_bwd(1, dx, None, bb, h, None, one, one, r1, r2, db, dres, None, dp, dq, scratch, n, d, n, 1.0, st)
torch.cuda.synchronize()
g = torch.cuda.CUDAGraph()
with torch.cuda.graph(g, stream=stream):
    step(stream.cuda_stream)
g.replay()
torch.cuda.synchronize()
a = [t.clone() for t in (h, y, dx, dw, db, dres, dp, dq)]
step(torch.cuda.current_stream().cuda_stream)
torch.cuda.synchronize()
assert all(torch.equal(p, q) for p, q in zip(a, (h, y, dx, dw, db, dres, dp, dq))) and float(dw.float().abs().max()) > 0.1
"""


@gpu
def test_first_call_of_a_process_may_be_a_recorded_one(binding):
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    r = subprocess.run([sys.executable, "-c", FIRST_CALL_IS_RECORDED], cwd=root, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stderr[-2000:]


# ---- refusals without a GPU -----------------------------------------------------------------------------------------
def test_act8_refusals(binding):
    assert [binding.act8_pitch(c) for c in (0, -1, 1, 16, 17, 131072, 131073)] == [0, 0, 16, 16, 32, 131072, 0]
    for fn in (binding.act8_pack, binding.act8_unpack):
        ok = dict(prec=1, x=P, q=P, s=P, rows=3, C=64)
        call = lambda **kw: status(fn, *{**ok, **kw}.values())  # noqa: E731, B023
        assert call(prec=2) == 1 and call(x=None) == 1 and call(q=None) == 1 and call(s=None) == 1
        assert call(rows=0) == 3 and call(C=0) == 3 and call(C=131073) == 3 and call(rows=-1) == 3
    assert status(binding.act8_pack, 1, P, P + 8, P, 3, 64) == 1 and status(binding.act8_unpack, 1, P + 8, P, P, 3, 64) == 1


def test_fc8_refusals(binding):
    need = binding.fc8_workspace_bytes(1, 4, 64, 100)
    assert need > 0
    for bad in ((2, 4, 64, 100), (1, 0, 64, 100), (1, 4, 0, 100), (1, 4, 64, 0), (1, 4, 131073, 100), (1, 4, 64, (1 << 24) + 1), (1, (1 << 24) + 1, 64, 100)):
        assert binding.fc8_workspace_bytes(*bad) == 0
    ok = dict(prec=1, xq=P, xs=P, wq=P, ws=P, bias=None, y=P, B=4, n_in=64, n_out=100)
    fwd = lambda **kw: status(binding.fc8_fwd, *{**ok, **kw}.values())  # noqa: E731
    assert fwd(prec=2) == 1 and fwd(prec=-1) == 1
    for name in ("xq", "xs", "wq", "ws", "y"):
        assert fwd(**{name: None}) == 1
    for name in ("B", "n_in", "n_out"):
        assert fwd(**{name: 0}) == 3 and fwd(**{name: -5}) == 3 and fwd(**{name: 1 << 25}) == 3
    assert fwd(xq=P + 8) == 1 and fwd(wq=P + 4) == 1
    okb = dict(prec=1, dy=P, xq=P, xs=P, wq=P, ws=P, dx=2 * P, dw=P, db=None, work=Ws(need), B=4, n_in=64, n_out=100)
    bwd = lambda **kw: status(binding.fc8_bwd, *{**okb, **kw}.values())  # noqa: E731
    for name in ("dy", "xq", "xs", "wq", "ws", "work"):
        assert bwd(**{name: None}) == 1
    assert bwd(dx=None, dw=None) == 1 and bwd(dx=P) == 1 and bwd(work=Ws(need - 1)) == 1 and bwd(work=Ws(need, P + 16)) == 1
    assert b"workspace" in binding.lib().ddg_last_error(None)
    assert bwd(B=0) == 3 and bwd(prec=7) == 1 and bwd(xq=P + 8) == 1 and bwd(wq=P + 8) == 1


def test_block_norm_refusals(binding):
    ok = dict(prec=1, b=P, res=P, gate=None, post=P, pre=P, h=P, y=2 * P, q=None, s=None, r1=None, r2=None, rows=3, C=256, span=3, alpha=1.0, eps=1e-6)
    fwd = lambda **kw: status(binding.block_norm_fwd, *{**ok, **kw}.values())  # noqa: E731
    assert fwd(prec=3) == 1 and fwd(y=None) == 1 and fwd(q=P) == 1 and fwd(s=P) == 1 and fwd(q=P + 8, s=P) == 1
    for name in ("b", "res", "post", "pre", "h"):
        assert fwd(**{name: None}) == 1
    assert fwd(eps=-1.0) == 1 and fwd(eps=NAN) == 1 and fwd(eps=INF) == 1 and fwd(alpha=INF) == 1 and fwd(alpha=NAN) == 1
    assert fwd(h=2 * P) == 1                                        # y over h
    assert fwd(rows=0) == 3 and fwd(C=0) == 3 and fwd(C=16385) == 3 and fwd(rows=(1 << 30) + 1) == 3 and fwd(span=0) == 3
    okb = dict(prec=1, dy=P, dh=None, b=P, h=P, gate=P, post=P, pre=P, r1=P, r2=P, db=P, dres=2 * P, dg=P, dpost=P, dpre=P, scratch=P, rows=3, C=256, span=3, alpha=1.0)
    bwd = lambda **kw: status(binding.block_norm_bwd, *{**okb, **kw}.values())  # noqa: E731
    for name in ("dy", "b", "h", "post", "pre", "r1", "r2", "db", "dres", "dpost", "dpre", "scratch"):
        assert bwd(**{name: None}) == 1
    assert bwd(gate=None) == 1 and bwd(dres=P) == 1 and bwd(alpha=NAN) == 1
    assert bwd(rows=0) == 3 and bwd(C=16385) == 3 and bwd(span=0) == 3
    assert binding.block_norm_scratch_elems(0, 8, 1) == 0 and binding.block_norm_scratch_elems(2, 16385, 1) == 0 and binding.block_norm_scratch_elems(2, 8, 0) == 0
    assert binding.block_norm_scratch_elems(2, 8, 2) > 0


def test_block8_refuses_tensors_off_their_values_boundaries(binding):
    """An address that is no multiple of the value's size would fault in the kernels."""
    need = binding.fc8_workspace_bytes(0, 4, 64, 100)
    calls = [
        (binding.act8_pack, dict(x=P, q=P, s=P), (3, 64), "x", "s"),
        (binding.act8_unpack, dict(q=P, s=P, x=P), (3, 64), "x", "s"),
        (binding.fc8_fwd, dict(xq=P, xs=P, wq=P, ws=P, bias=P, y=P), (4, 64, 100), "bias y", "xs ws"),
        (binding.fc8_bwd, dict(dy=P, xq=P, xs=P, wq=P, ws=P, dx=2 * P, dw=3 * P, db=P, work=Ws(need)), (4, 64, 100), "dy dx dw", "xs ws db"),
        (binding.block_norm_fwd, dict(b=P, res=P, gate=P, post=P, pre=P, h=P, y=2 * P, q=4 * P, s=P, r1=P, r2=P), (3, 256, 3), "b res gate post pre h y", "s r1 r2"),
        (binding.block_norm_bwd, dict(dy=P, dh=P, b=P, h=P, gate=P, post=P, pre=P, r1=P, r2=P, db=P, dres=2 * P, dg=P, dpost=P, dpre=P, scratch=P), (3, 256, 3),
         "dy dh b h gate post pre db dres", "r1 r2 dg dpost dpre scratch"),
    ]
    for fn, args, sizes, elems, words in calls:
        for prec in (0, 1):
            for name in elems.split() + words.split():
                off = (1,) if prec and name in elems.split() else (1, 2, 3)
                for by in off:
                    kw = {**args, name: args[name] + by}
                    assert status(fn, prec, *kw.values(), *sizes) == 1, (fn.__name__, name, prec, by)
                    assert b"boundary" in binding.lib().ddg_last_error(None)
    # 32-bit results of 16-bit layers
    assert status(binding.fc8_fwd, 1, P, P, P, P, None, P + 2, 4, 64, 100, True) == 1
    assert status(binding.fc8_bwd, 1, P, P, P, P, P, None, P + 2, None, Ws(need), 4, 64, 100, True) == 1


def test_block8_refuses_outputs_over_what_other_blocks_read(binding):
    last = lambda: binding.lib().ddg_last_error(None)  # noqa: E731
    assert status(binding.act8_pack, 1, P, P, P, 3, 64) == 1 and b"may not be x" in last()
    assert status(binding.act8_unpack, 1, P, P, P, 3, 64) == 1 and b"may not be x" in last()
    need = binding.fc8_workspace_bytes(1, 64, 64, 64)
    bwd = lambda dx, dw: status(binding.fc8_bwd, 1, P, P, P, P, P, dx, dw, None, Ws(need), 64, 64, 64)  # noqa: E731
    assert bwd(2 * P, P) == 1 and b"dW" in last() and bwd(None, P) == 1 and bwd(2 * P, 2 * P) == 1 and b"dW" in last()
    for over in range(4):
        t = [2 * P, 3 * P, 4 * P, 5 * P]  # b, res, h, y
        t[over] = P
        assert status(binding.block_norm_fwd, 1, t[0], t[1], None, P, P, t[2], t[3], P, P, None, None, 3, 256, 3) == 1 and b"place of their own" in last()


def test_block8_tensor_arguments_are_checked_in_the_binding(binding):
    x, q = torch.zeros(4, 8), torch.zeros(4, 16, dtype=torch.int8)
    for bad in (dict(x=x.t()), dict(x=x.half()), dict(x=x[:2]), dict(q=q[:, :8]), dict(q=q.float()), dict(q=q[:3])):
        a = {**dict(x=x, q=q), **bad}
        with pytest.raises(ValueError):
            binding.act8_pack(0, a["x"], a["q"], P, 4, 8)


# ---- bounded waits --------------------------------------------------------------------------------------------------
# every way of a call that waits on the device: one row, a few, tiles, with splits, with chains that are cut, fp32
WAYS_THAT_WAIT = [(1, 4096, 700, 1), (20, 2048, 300, 1), (100, 4096, 640, 1), (300, 136, 777, 1), (700, 2200, 1100, 1), (300, 8200, 70, 1), (2100, 264, 1000, 0), (130, 72, 2057, 0), (2200, 1000, 2300, 1), (2200, 2300, 1000, 1),
                 (300, 2300, 2200, 1)]


@gpu
@pytest.mark.parametrize("shape", WAYS_THAT_WAIT, ids=ids)
def test_fc8_waits_that_run_out(binding, shape):
    """With limits of few polls and of none, each kernel lets its copies and products land and returns; what was not computed is
    NaN, the rest the usual bits; the calls after it are not touched."""
    c = Fc(*shape, bias=True, seed=51)
    step = lambda: [c.fwd(binding)] + [t for f in (False, True) for t in c.bwd(binding, "xw", f)[:2]]  # noqa: E731
    ref = step()
    try:
        for polls in (0, 1, 2, 1, 4, 1, 8, 16, 50, 400, 0):
            binding.debug_block8_wait_polls(polls)
            got = step()
            torch.cuda.synchronize()
            for a, b in zip(got, ref):
                lost = torch.isnan(a)
                assert torch.equal(torch.where(lost, b, a), b)
                assert polls > 0 or bool(lost.all())
    finally:
        binding.debug_block8_wait_polls(-1)
    assert all(torch.equal(a, b) for a, b in zip(step(), ref))


@gpu
@PREC
@pytest.mark.parametrize("rows,C", [(400, 2048), (320, 1021), (3000, 640)])
def test_rows_through_shared_memory_whose_waits_run_out(binding, rows, C, prec):
    """Without a poll every row is NaN, its codes too; the calls after it are not touched."""
    c = Norm(rows, C, prec, 100, seed=52).reference()
    h, r1, r2 = c.h.to(DT[prec]), c.r1[:, 0].float(), c.r2[:, 0].float()
    step = lambda: list(c.fwd(binding, True, False)[:2]) + [c.fwd(binding, False, True)[3]] + list(c.bwd(binding, h, r1, r2)) + [pack(binding, c.b, prec)[1]]  # noqa: E731
    ref = step()
    try:
        binding.debug_block8_wait_polls(0)
        got = step()
        torch.cuda.synchronize()
        for a, b in zip(got, ref):  # (narrow rows of bf16 are a warp's, which waits for nothing, in some of the calls)
            lost = bool(torch.isnan(a).all())
            assert lost or (C == 640 and torch.equal(a, b))
    finally:
        binding.debug_block8_wait_polls(-1)
    assert all(torch.equal(a, b) for a, b in zip(step(), ref))


@gpu
@PREC
@pytest.mark.parametrize("rows,C,span", [(320, 1021, 320), (3000, 640, 7), (900, 4096, 1), (8192, 4096, 8192)])
def test_rows_through_shared_memory_whose_waits_run_out_in_some_threads(binding, rows, C, span, prec):
    """With limits of a few polls a row may have come for some threads of its block and not for others, most of all while other
    work keeps the memory busy: every value is NaN or the usual bits, sums included, and a row is NaN as a whole."""
    c = Norm(rows, C, prec, span, seed=56).reference()
    h, r1, r2 = c.h.to(DT[prec]), c.r1[:, 0].float(), c.r2[:, 0].float()
    side, busy = torch.cuda.Stream(), torch.empty(2, 1 << 30, dtype=torch.uint8, device="cuda")

    def step():
        to_codes = c.fwd(binding, False, True)
        return list(c.bwd(binding, h, r1, r2)) + list(c.fwd(binding, True, False)[:2]) + [to_codes[0], to_codes[3], pack(binding, c.b, prec)[1]]

    ref = step()
    try:
        for polls in (1,) * 40 + (2, 3, 4, 8):
            binding.debug_block8_wait_polls(polls)
            torch.cuda.synchronize()
            with torch.cuda.stream(side):
                busy[0].copy_(busy[1])
                busy[1].copy_(busy[0])
            got = step()
            torch.cuda.synchronize()
            for k, (a, b) in enumerate(zip(got, ref)):
                lost = torch.isnan(a)
                assert torch.equal(torch.where(lost, b, a), b), (polls, k)
                if k in (0, 1, 5, 6, 7):  # db, dres, h, y, h
                    assert torch.equal(lost.all(1), lost.any(1)), (polls, k)
            # a block that lost a row has a share in the sums over all rows
            assert not torch.isnan(got[0]).any() or (torch.isnan(got[3]).all() and torch.isnan(got[4]).all()), polls
    finally:
        binding.debug_block8_wait_polls(-1)
    assert all(torch.equal(a, b) for a, b in zip(step(), ref))


# ---- rows through shared memory: as the tests of few rows above -----------------------------------------------------------
@gpu
@PREC
@pytest.mark.parametrize("rows,C,span", [(2000, 640, 1), (1000, 4096, 1), (1500, 1021, 2), (900, 1536, 2), (400, 8192, 1), (2300, 512, 1), (601, 3000, 5)])
def test_block_norm_several_stretches_of_a_block(binding, rows, C, span, prec):
    """More gates than resident blocks: a block's share of dgamma_post comes out of several stretches."""
    for dh in (True, False):
        c = Norm(rows, C, prec, span, seed=62).reference()
        h, r1, r2 = c.h.to(DT[prec]), c.r1[:, 0].float(), c.r2[:, 0].float()
        got, refs = c.bwd(binding, h, r1, r2, dh), c.grads_ref(h, r1, r2, dh)
        for g, (ref, tol), what in zip(got, refs, ("db", "dres", "dgate", "dgamma_post", "dgamma_pre")):
            within(g, ref, tol, what)
        again = c.bwd(binding, h, r1, r2, dh, dgate=False)
        assert all(torch.equal(a, b) for k, (a, b) in enumerate(zip(got, again)) if k != 2)
    got, y, q, s, _, _ = c.fwd(binding, True, True)
    within(got, c.h, c.e_h + U[h.dtype] * c.h.abs(), "h")
    within(y, c.y, c.e_y + U[h.dtype] * c.y.abs(), "y")
    within(q[:, :C].double() * s.double()[:, None], c.y, s.double()[:, None] * (0.5 + 2.0 ** -12) + 2 * c.e_y.amax(1, keepdim=True), "codes")


@gpu
@PREC
@pytest.mark.parametrize("rows,C,span", [(700, 640, 100), (400, 1021, 7), (601, 2933, 1), (320, 4096, 320)])
def test_block_norm_of_many_rows_in_place(binding, rows, C, span, prec):
    """h and y over b and res; db and dres over what the backward pass reads; rows whose 16-byte units are shared too."""
    c = Norm(rows, C, prec, span, seed=63).reference()
    h, y, _, _, r1, r2 = c.fwd(binding)
    for a, b in (("b", "res"), ("res", "b")):
        k = Norm(rows, C, prec, span, seed=63)
        h2, y2, _, _, _, _ = k.fwd(binding, h=getattr(k, a), y=getattr(k, b))
        assert torch.equal(h2, h) and torch.equal(y2, y)
    ref = c.bwd(binding, h, r1, r2)
    for a, b in (("dy", "dh"), ("dh", "b"), ("b", "dy"), ("h", "dh"), ("b", "h"), ("h", "dy")):
        k = Norm(rows, C, prec, span, seed=63)
        k.h = h.clone()
        got = k.bwd(binding, k.h, r1, r2, db=getattr(k, a), dres=getattr(k, b))
        assert all(torch.equal(p, q) for p, q in zip(got, ref)), (a, b)


@gpu
@PREC
@pytest.mark.parametrize("C", [640, 1021, 2048])
def test_block_norm_special_rows_among_many(binding, C, prec):
    """Rows of zeros, NaN and infinities are their own, in the gradients too; sums over rows show them."""
    rows = 400
    c = Norm(rows, C, prec, 1, seed=64)
    clean = c.fwd(binding, True, True)
    clean_grads = c.bwd(binding, clean[0], clean[4], clean[5])
    c.b[1], c.res[1] = 0.0, 0.0
    c.b[200, 7], c.res[399, C - 1], c.b[0, 0] = NAN, INF, -INF
    c.gate[40] = 0.0
    h, y, q, s, r1, r2 = c.fwd(binding, True, True)
    assert not h[1].any() and not y[1].any() and not q[1].any() and float(s[1]) == 2.0 ** -126
    for r in (200, 399, 0):
        assert math.isnan(float(s[r])) and not q[r].any()
    assert torch.isnan(y[200]).all()
    assert torch.equal(h[40], (ALPHA * c.res[40].float()).to(h.dtype))
    same = torch.ones(rows, dtype=torch.bool, device="cuda")
    same[[0, 1, 40, 200, 399]] = False
    for a, b in zip((h, y, q, s, r1, r2), clean):
        assert torch.equal(a[same], b[same])
    db, dres, dg, dpost, dpre = c.bwd(binding, h, r1, r2)
    for a, b in zip((db, dres, dg), clean_grads):
        assert torch.equal(a[same], b[same]) and torch.isnan(a[200].float()).all() and torch.isfinite(a[[1, 40]].float()).all()
    assert torch.isnan(dpost).all() and torch.isnan(dpre).all()


@gpu
@PREC
@pytest.mark.parametrize("C", [1021, 2048, 8192])
def test_act8_special_rows_among_many(binding, C, prec):
    rows = 320
    x = randn(rows, C, seed=65, prec=prec)
    clean = pack(binding, x, prec)
    x[1] = 0.0
    x[2] = randn(C, seed=5, prec=prec) * 2.0 ** -130
    x[3, 7] = torch.finfo(x.dtype).max
    x[4, 9], x[300, 3], x[319, C - 1], x[0, 0] = NAN, INF, -INF, NAN
    q, scale = pack(binding, x, prec)
    bad = [0, 4, 300, 319]
    for r in bad:
        assert math.isnan(float(scale[r])) and not q[r].any()
    good = [r for r in range(rows) if r not in bad]
    ref, s = codes(x[good])
    assert torch.equal(q[good][:, :C].double(), ref) and torch.equal(scale[good], s)
    back = torch.empty_like(x)
    binding.act8_unpack(prec, q, scale, back, rows, C)
    assert torch.isnan(back[bad]).all() and torch.isfinite(back[good]).all() and not back[1].any()
    assert torch.equal(q[5:300], clean[0][5:300]) and torch.equal(scale[5:300], clean[1][5:300])


@gpu
@PREC
def test_many_rows_off_16_byte_boundaries_and_rows_behind(binding, prec):
    """Tensors that start anywhere, one at a time and all; rows behind the last are left as they were."""
    def off(t):
        store = torch.empty(t.numel() + 1, dtype=t.dtype, device="cuda")
        store[1:] = t.flatten()
        return store[1:].view(t.shape)
    for rows, C in ((330, 1024), (310, 1021)):
        names = ("b", "res", "gate", "post", "pre", "dy", "dh")
        for which in [(n,) for n in names] + [names]:
            c = Norm(rows, C, prec, 10, seed=66).reference()
            for n in which:
                setattr(c, n, off(getattr(c, n)))
            h, y, q, s, r1, r2 = c.fwd(binding, True, True)
            within(h, c.h, c.e_h + U[h.dtype] * c.h.abs(), "h")
            within(y, c.y, c.e_y + U[h.dtype] * c.y.abs(), "y")
            for g, (ref, tol), what in zip(c.bwd(binding, h, r1, r2), c.grads_ref(h, r1, r2), ("db", "dres", "dgate", "dgamma_post", "dgamma_pre")):
                within(g, ref, tol, what)
        # fewer rows than the buffers have
        n = rows - 3
        h, y, db, dres, q, s = (torch.full_like(t, 7.0) for t in (c.b, c.b, c.b, c.b, q, s))
        binding.block_norm_fwd(prec, c.b, c.res, c.gate, c.post, c.pre, h, y, q, s, r1, r2, n, C, 10, ALPHA, EPS)
        dg, dpost, dpre, scratch = f32(*c.gate.shape), f32(C), f32(C), f32(binding.block_norm_scratch_elems(n, C, 10) + 64)
        binding.block_norm_bwd(prec, c.dy, c.dh, c.b, h, c.gate, c.post, c.pre, r1, r2, db, dres, dg, dpost, dpre, scratch, n, C, 10, ALPHA)
        assert all((t[n:] == 7).all() for t in (h, y, db, dres, q, s)) and (scratch[-64:] == 7).all()
        assert not any((t[:n] == 7).all(1).any() for t in (h, y, db, dres))
        q2, s2 = torch.full_like(q, 7), f32(rows)
        binding.act8_pack(prec, c.b, q2, s2, n, C)
        assert (q2[n:] == 7).all() and (s2[n:] == 7).all()
        ref, sr = codes(c.b[:n])
        assert torch.equal(q2[:n, :C].double(), ref) and torch.equal(s2[:n], sr)


# ---- long sums, large tensors ---------------------------------------------------------------------------------------
@gpu
def test_fc8_weight_gradient_of_many_rows_keeps_its_precision(binding):
    """Products of one sign, whose truncated sums drift most: chains are cut after 1024 products for fp32 results (6.6e-7 of the
    sum each) and after 65536 for bf16 ones (1.5e-4), the pieces added rounded to nearest."""
    for B, dw_f32, tol in ((20000, True, 1e-6), (200000, False, 2.0 ** -8 + 2e-4)):
        D, V = 48, 40
        c = Fc(B, D, V, 1, seed=53)
        c.xq.fill_(101), c.xs.fill_(2.0 ** -6), c.dy.fill_(1.25)
        dw = c.bwd(binding, "w", dw_f32)[1]
        ref = B * 1.25 * 101 * 2.0 ** -6
        assert float(((dw.double() - ref).abs() / ref).max()) <= tol
    c = Fc(40, 64, 30000, 1, seed=54)
    c.wq.fill_(101), c.ws.fill_(2.0 ** -6), c.dy.fill_(1.25)
    dx = c.bwd(binding, "x")[0]
    ref = 30000 * 1.25 * 101 * 2.0 ** -6
    assert float(((dx.double() - ref).abs() / ref).max()) <= 2.0 ** -8 + 2e-4


@gpu
def test_offsets_past_32_bits(binding):
    """Tensors of more than 2^31 values: what stands at their ends."""
    B, D, V = 33100, 96, 65536
    c = Fc(300, D, V, 1, seed=55)
    xq, xs = c.xq.repeat(111, 1)[:B].contiguous(), c.xs.repeat(111)[:B].contiguous()
    y = torch.empty(B, V, dtype=torch.bfloat16, device="cuda")
    binding.fc8_fwd(1, xq, xs, c.wq, c.ws, None, y, B, D, V)
    last = torch.arange(B - 200, B, device="cuda")
    full, tol = c.y_ref(U[torch.bfloat16])
    within(y[last], full[last % 300], tol[last % 300], "y")
    # the same tensor as dy
    ws = torch.empty(binding.fc8_workspace_bytes(1, B, D, V), dtype=torch.uint8, device="cuda")
    dx = torch.empty(B, D, dtype=torch.bfloat16, device="cuda")
    binding.fc8_bwd(1, y, None, None, c.wq, c.ws, dx, None, None, ws, B, D, V)
    w = value(c.wq, c.ws, D, 1).double()
    d = y[last].double()
    within(dx[last], d @ w, (4 * math.ceil(V / 16) + 16) * E * (d.abs() @ w.abs()) + U[torch.bfloat16] * (d @ w).abs(), "dx")
    del ws, dx, d
    # as rows to codes, and rows of norms: C = 16384
    C = 16384
    rows = B * V // C
    x = y.view(-1)[: rows * C].view(rows, C)
    q, s = pack(binding, x, 1)
    tail = slice(rows - 40, rows)
    ref, sr = codes(x[tail])
    assert torch.equal(q[tail].double(), ref) and torch.equal(s[tail], sr)
    back = torch.empty_like(x)
    binding.act8_unpack(1, q, s, back, rows, C)
    assert torch.equal(back[tail], value(q[tail], s[tail], C, 1))
    del q
    one = torch.ones(C, dtype=torch.bfloat16, device="cuda")
    r1, r2 = f32(rows), f32(rows)
    h = torch.empty_like(x)
    binding.block_norm_fwd(1, x, back, None, one, one, h, back, None, None, r1, r2, rows, C, rows, 0.0, EPS)
    n = x[tail].double()
    n = n / (n.square().mean(1, keepdim=True) + EPS).sqrt()
    within(h[tail], n, (RSTD_E + 4 * E + U[torch.bfloat16]) * n.abs() * 1.01 + 1e-30, "h")
    dp, dq = f32(C), f32(C)
    scratch = f32(binding.block_norm_scratch_elems(rows, C, rows))
    binding.block_norm_bwd(1, back, None, x, h, None, one, one, r1, r2, back, x, None, dp, dq, scratch, rows, C, rows, 0.0)
    assert not x[tail].any() and torch.isfinite(back[tail].float()).all() and torch.isfinite(dq).all()

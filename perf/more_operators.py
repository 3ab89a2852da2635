"""Measured cases of the operators around a linear layer that works and keeps its activations in 8 bits: the norms before
and after a block with its gate and residual scale, rows of 8-bit codes with a scale each (activation checkpoints), and the
linear layer whose product runs on such codes and whose backward pass reads them.  `own` chooses between the operators'
plain forms (elementary torch operations in 32 bits) and the library's kernels.

A case has a `kind`:
  norm_serve    norm after a block, gate, residual scale, norm before the next block
  norm_train    the same with its backward pass
  linear_serve  the same norms, their result as 8-bit codes, and the product of the codes with those of a weight
  product       product of 8-bit codes with a scale for each token and channel
  checkpoint    rows to 8-bit codes and back
  linear_train  a training step of the linear layer: activations and weight to codes, product, and the gradients from the
                codes that were kept

Codes are kept in rows of a multiple of 16 bytes, zeros behind the row's own.
"""
import math

import torch

own = False

_DT = {"bf16": torch.bfloat16, "fp32": torch.float32}
_EPS = 1e-6
_LEAST = 127.0 * 2.0 ** -126  # a row's maximum counts as at least this: its scale stays a normal number


def listed():
    return [
        # one token between two blocks: latency
        _norm("norm_serve_one_row", "norm_serve", 1, 4096, "bf16"),
        # seven samples with a gate each, odd sizes, 32 bits
        _norm("norm_train_fp32", "norm_train", 777, 1021, "fp32", span=111),
        # training, ordinary width, one gate vector
        _norm("norm_train", "norm_train", 8192, 4096, "bf16"),
        # decoding, one token: bound by reading the weight's codes
        _linear("serve_one_token", "linear_serve", 1, 4096, 16384, "bf16"),
        # decoding a small batch, sizes that fill no tile
        _linear("serve_ragged", "linear_serve", 37, 1000, 5001, "bf16", bias=True),
        # a prompt
        _linear("serve_prompt", "linear_serve", 4096, 4096, 4096, "bf16"),
        # a long prompt through the wide layer of a large model, codes in hand
        _linear("product_large", "product", 16384, 4096, 16384, "bf16"),
        # hidden layer of the multilayer perceptron at batch 128: one slot of the activation history
        _linear("checkpoint_small", "checkpoint", 128, 128, 0, "fp32"),
        # activations of a large layer
        _linear("checkpoint_large", "checkpoint", 8192, 8192, 0, "bf16"),
        # hidden layer of the multilayer perceptron at batch 128, training
        _linear("train_small", "linear_train", 128, 128, 128, "bf16", bias=True, wide=True),
        # ragged in every size, 32 bits
        _linear("train_fp32", "linear_train", 1111, 520, 2007, "fp32", bias=True),
        # wide layer of a large model, gradients as the update reads them
        _linear("train_large", "linear_train", 8192, 4096, 16384, "bf16", wide=True),
    ]


def _norm(name, kind, rows, width, dtype, span=0):
    """span: rows that share a row of the gate, 0: all."""
    return {"name": name, "kind": kind, "rows": rows, "width": width, "dtype": dtype, "span": span or rows}


def _linear(name, kind, rows, width, out, dtype, bias=False, wide=False):
    """wide: the result of a product alone, or the weight's gradient (training), in 32 bits whatever the type."""
    return {"name": name, "kind": kind, "rows": rows, "width": width, "out": out, "dtype": dtype, "bias": bias, "wide": wide}


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["norm_serve", "norm_train", "linear_serve", "linear_serve", "product", "checkpoint", "linear_train", "linear_train"])
    dtype = rng.choice(["bf16", "bf16", "bf16", "fp32"])
    width = _log(rng, 64, 8192)
    if rng.random() < 0.7:
        width = -(-width // 64) * 64
    if kind.startswith("norm"):
        span, gates = _log(rng, 1, 8192), rng.choice([1, 1, 2, 3, 16])
        while span * gates * width > 8192 * 4096:
            span = span // 2 or 1
        c = _norm("", kind, span * gates, width, dtype, span)
    elif kind == "checkpoint":
        rows = _log(rng, 1, 16384)
        while rows * width > 8192 * 8192:
            rows //= 2
        c = _linear("", kind, rows, width, 0, dtype)
    else:
        rows, out = _log(rng, 1, 8192), _log(rng, 64, 16384)
        if rng.random() < 0.7:
            out = -(-out // 64) * 64
        # serving calls of many rows are as common as those of a few
        if kind != "linear_train" and rng.random() < 0.5:
            rows = _log(rng, 1, 128)
        # a serving call between two norms works and answers in 16 bits; 32-bit gradients take three products each
        if kind == "linear_serve":
            dtype = "bf16"
        elif dtype == "fp32":
            rows = min(rows, 2048)
        width = min(width, 4096)
        c = _linear("", kind, rows, width, out, dtype, rng.random() < 0.3, dtype == "bf16" and kind != "linear_serve" and rng.random() < 0.4)
    del c["name"]
    return c


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    dt, kind, n, d = _DT[case["dtype"]], case["kind"], case["rows"], case["width"]

    def normal(*size, std=1.0, mean=0.0):
        return torch.empty(size, device="cuda", dtype=dt).normal_(mean, std, generator=g)

    s = {"case": case, "kind": kind}
    if kind.startswith("norm") or kind == "linear_serve":
        # a residual stream is wider than what a block adds to it; weights of the norms near one, gates learned from small ones
        span = case.get("span", n)
        s |= {"b": normal(n, d), "res": normal(n, d, std=3.0), "gate": normal(n // span, d, std=0.2, mean=0.5), "span": span, "alpha": 0.875,
              "post": normal(d, std=0.1, mean=1.0), "pre": normal(d, std=0.1, mean=1.0)}
    if kind == "norm_train":
        s |= {"dy": normal(n, d), "dh": normal(n, d)}
    if kind in ("checkpoint", "linear_train"):
        # tokens of unlike size
        s["x"] = normal(n, d) * (0.5 + torch.rand(n, 1, device="cuda", generator=g)).to(dt)
    if kind == "linear_train":
        s |= {"w": normal(case["out"], d, std=1.0 / math.sqrt(d)), "dy": normal(n, case["out"])}
    if kind in ("linear_serve", "product"):
        # the weight, and for a product alone the tokens, as codes that were written before
        s["wq"], s["ws"] = _random_codes(case["out"], d, 1.0 / math.sqrt(d), g)
        if kind == "product":
            s["xq"], s["xs"] = _random_codes(n, d, 1.0, g)
    if kind not in ("norm_serve", "norm_train", "checkpoint"):
        s["bias"] = normal(case["out"]) if case["bias"] else None
    return s


def _random_codes(rows, cols, std, g):
    """Codes and scales of rows of normal values."""
    v = torch.empty(rows, cols, device="cuda").normal_(0.0, std, generator=g)
    q, scale = _to_codes(v)
    kept = torch.zeros(rows, -(-cols // 16) * 16, device="cuda", dtype=torch.int8)
    kept[:, :cols] = q.to(torch.int8)
    return kept, scale


def run(state):
    kind = state["kind"]
    if own:
        return {"norm_serve": _own_norm_serve, "norm_train": _own_norm_train, "linear_serve": _own_linear_serve, "product": _own_product,
                "checkpoint": _own_checkpoint, "linear_train": _own_linear_train}[kind](state)
    return {"norm_serve": _norm_serve, "norm_train": _norm_train, "linear_serve": _linear_serve, "product": _product,
            "checkpoint": _checkpoint, "linear_train": _linear_train}[kind](state)


# ---- plain forms ---------------------------------------------------------------------------------------------------
def _to_codes(v):
    """Whole numbers of -127 to 127 for each row, and the row's scale; in 64 bits, for values at the border of two codes."""
    top = v.abs().amax(1, keepdim=True).clamp(min=_LEAST)
    return (v.double() * 127.0 / top.double()).round().float(), (top / 127.0)[:, 0]


def _per_row(gate, span):
    """The gate of every row."""
    return gate.float().repeat_interleave(span, 0)


def _normed(s):
    b = s["b"].float()
    r1 = torch.rsqrt(b.square().mean(1, keepdim=True) + _EPS)
    h = s["alpha"] * s["res"].float() + _per_row(s["gate"], s["span"]) * (b * r1 * s["post"].float())
    r2 = torch.rsqrt(h.square().mean(1, keepdim=True) + _EPS)
    return h, h * r2 * s["pre"].float(), r1, r2


def _norm_serve(s):
    h, y, _, _ = _normed(s)
    dt = s["b"].dtype
    return {"h": h.to(dt), "y": y.to(dt)}


def _norm_train(s):
    dt, span = s["b"].dtype, s["span"]
    h, y, r1, r2 = _normed(s)
    # the backward pass has the sum as it was stored
    kept, b, dy, pre, post, gate = h.to(dt).float(), s["b"].float(), s["dy"].float(), s["pre"].float(), s["post"].float(), _per_row(s["gate"], span)
    wdy = dy * pre
    t = s["dh"].float() + r2 * (wdy - kept * (r2 * r2) * (wdy * kept).mean(1, keepdim=True))
    unit = b * r1
    du = gate * t
    wdu = du * post
    db = r1 * (wdu - b * (r1 * r1) * (wdu * b).mean(1, keepdim=True))
    return {"h": h.to(dt), "y": y.to(dt), "db": db.to(dt), "dres": (s["alpha"] * t).to(dt), "dgate": (t * unit * post).view(-1, span, b.shape[1]).sum(1),
            "dpost": (du * unit).sum(0), "dpre": (dy * kept * r2).sum(0)}


def _scaled_product(xq, xs, wq, ws, bias):
    y = (xq @ wq.t()) * xs[:, None] * ws
    return y if bias is None else y + bias.float()


def _linear_serve(s):
    d, dt = s["b"].shape[1], s["b"].dtype
    h, y, _, _ = _normed(s)
    q, scale = _to_codes(y)
    z = _scaled_product(q, scale, s["wq"][:, :d].float(), s["ws"], s["bias"])
    return {"h": h.to(dt), "z": z.to(dt)}


def _product(s):
    d, dt = s["case"]["width"], _DT[s["case"]["dtype"]]
    z = _scaled_product(s["xq"][:, :d].float(), s["xs"], s["wq"][:, :d].float(), s["ws"], s["bias"])
    return {"z": z if s["case"]["wide"] else z.to(dt)}


def _checkpoint(s):
    q, scale = _to_codes(s["x"].float())
    return {"x": (q * scale[:, None]).to(s["x"].dtype), "scale": scale}


def _linear_train(s):
    x, w, dt = s["x"], s["w"], s["x"].dtype
    (xq, xs), (wq, ws) = _to_codes(x.float()), _to_codes(w.float())
    z = _scaled_product(xq, xs, wq, ws, s["bias"])
    # the backward pass has both operands as their codes stand for them, in the tensors' type
    dy, x, w = s["dy"].float(), (xq * xs[:, None]).to(dt).float(), (wq * ws[:, None]).to(dt).float()
    dw = dy.t() @ x
    out = {"z": z.to(dt), "dx": (dy @ w).to(dt), "dw": dw if s["case"]["wide"] else dw.to(dt)}
    if s["bias"] is not None:
        out["db"] = dy.sum(0)
    return out


# ---- the library's kernels -----------------------------------------------------------------------------------------
def _prec(t):
    return 1 if t.dtype == torch.bfloat16 else 0


def _f32(*size):
    return torch.empty(size, dtype=torch.float32, device="cuda")


def _stream():
    return torch.cuda.current_stream().cuda_stream


def _own_norm_fwd(s, to_codes=False, keep=False):
    from paper_1804_10574_b200 import binding
    b = s["b"]
    n, d = b.shape
    h = torch.empty_like(b)
    y = None if to_codes else torch.empty_like(b)
    q, scale = (torch.empty((n, binding.act8_pitch(d)), dtype=torch.int8, device="cuda"), _f32(n)) if to_codes else (None, None)
    r1, r2 = (_f32(n), _f32(n)) if keep else (None, None)
    binding.block_norm_fwd(_prec(b), b, s["res"], s["gate"], s["post"], s["pre"], h, y, q, scale, r1, r2, n, d, s["span"], s["alpha"], _EPS, _stream())
    return h, y, q, scale, r1, r2


def _own_norm_serve(s):
    h, y, _, _, _, _ = _own_norm_fwd(s)
    return {"h": h, "y": y}


def _own_norm_train(s):
    from paper_1804_10574_b200 import binding
    b, gate = s["b"], s["gate"]
    n, d = b.shape
    h, y, _, _, r1, r2 = _own_norm_fwd(s, keep=True)
    db, dres, dgate, dpost, dpre = torch.empty_like(b), torch.empty_like(b), _f32(*gate.shape), _f32(d), _f32(d)
    scratch = _f32(binding.block_norm_scratch_elems(n, d, s["span"]))
    binding.block_norm_bwd(_prec(b), s["dy"], s["dh"], b, h, gate, s["post"], s["pre"], r1, r2, db, dres, dgate, dpost, dpre, scratch, n, d, s["span"], s["alpha"],
                           _stream())
    return {"h": h, "y": y, "db": db, "dres": dres, "dgate": dgate, "dpost": dpost, "dpre": dpre}


def _own_z(s, xq, xs, wq, ws, dt, wide):
    from paper_1804_10574_b200 import binding
    n, out = xq.shape[0], wq.shape[0]
    z = torch.empty((n, out), dtype=torch.float32 if wide else dt, device="cuda")
    binding.fc8_fwd(1 if dt == torch.bfloat16 else 0, xq, xs, wq, ws, s["bias"], z, n, s["case"]["width"], out, wide, _stream())
    return z


def _own_linear_serve(s):
    h, _, q, scale, _, _ = _own_norm_fwd(s, to_codes=True)
    return {"h": h, "z": _own_z(s, q, scale, s["wq"], s["ws"], h.dtype, False)}


def _own_product(s):
    return {"z": _own_z(s, s["xq"], s["xs"], s["wq"], s["ws"], _DT[s["case"]["dtype"]], s["case"]["wide"])}


def _own_pack(x):
    from paper_1804_10574_b200 import binding
    n, d = x.shape
    q, scale = torch.empty((n, binding.act8_pitch(d)), dtype=torch.int8, device="cuda"), _f32(n)
    binding.act8_pack(_prec(x), x, q, scale, n, d, _stream())
    return q, scale


def _own_checkpoint(s):
    from paper_1804_10574_b200 import binding
    x = s["x"]
    q, scale = _own_pack(x)
    back = torch.empty_like(x)
    binding.act8_unpack(_prec(x), q, scale, back, x.shape[0], x.shape[1], _stream())
    return {"x": back, "scale": scale}


def _own_linear_train(s):
    from paper_1804_10574_b200 import binding
    x, w, dy, wide = s["x"], s["w"], s["dy"], s["case"]["wide"]
    (n, d), out, p = x.shape, w.shape[0], _prec(x)
    (xq, xs), (wq, ws) = _own_pack(x), _own_pack(w)
    z = _own_z(s, xq, xs, wq, ws, x.dtype, False)
    dx, dw = torch.empty_like(x), torch.empty(w.shape, dtype=torch.float32 if wide else w.dtype, device="cuda")
    db = _f32(out) if s["bias"] is not None else None
    work_space = torch.empty(binding.fc8_workspace_bytes(p, n, d, out), dtype=torch.uint8, device="cuda")
    binding.fc8_bwd(p, dy, xq, xs, wq, ws, dx, dw, db, work_space, n, d, out, wide, _stream())
    got = {"z": z, "dx": dx, "dw": dw}
    if db is not None:
        got["db"] = db
    return got


# ---- work ----------------------------------------------------------------------------------------------------------
def work(case):
    e = 2 if case["dtype"] == "bf16" else 4
    kind, n, d = case["kind"], case["rows"], case["width"]
    if kind.startswith("norm"):
        gates = n // case["span"]
        if kind == "norm_serve":
            return {"bytes": 4 * n * d * e + (gates + 2) * d * e, "flops": 11 * n * d}
        # b and the sum are read again after all rows were written
        return {"bytes": 10 * n * d * e + (gates + 2) * d * (2 * e + 4), "flops": 40 * n * d}
    if kind == "checkpoint":
        return {"bytes": 2 * (n * d * (e + 1) + 4 * n), "flops": 5 * n * d}
    out = case["out"]
    flops, side = 2 * n * d * out, 4 * (n + out) + (out * e if case["bias"] else 0)
    result = n * out * (4 if case["wide"] or case["dtype"] == "fp32" else 2)
    if kind == "linear_serve":
        return {"bytes": 3 * n * d * e + 3 * d * e + out * d + result + side, "flops": flops + 13 * n * d}
    if kind == "product":
        return {"bytes": (n + out) * d + result + side, "flops": flops}
    grads = n * d * e + out * d * (4 if case["wide"] else e) + (4 * out if case["bias"] else 0)
    return {"bytes": (n + out) * d * e + 2 * n * out * e + side + grads, "flops": 3 * flops}


# ---- 64 bits -------------------------------------------------------------------------------------------------------
def exact(case, seed):
    s = prepare(case, seed)
    return {"norm_serve": _exact_norm, "norm_train": _exact_norm, "linear_serve": _exact_linear_serve, "product": _exact_product,
            "checkpoint": _exact_checkpoint, "linear_train": _exact_linear_train}[case["kind"]](case, s)


def _exact_rows(v):
    """What the codes of rows stand for, and the scales."""
    top = torch.linalg.vector_norm(v, ord=math.inf, dim=1, keepdim=True).clamp(min=_LEAST)
    # the code below, and by whole multiples of the values, which are exact, whether the next one is nearer; halves go to even
    low = torch.floor(127 * v / top)
    twice, border = 254 * v, (2 * low + 1) * top
    up = (twice > border) | ((twice == border) & (low % 2 != 0))
    return (low + up) * (top / 127), top[:, 0] / 127


def _exact_sum(case, s):
    b = s["b"].double()
    rms = (torch.linalg.vector_norm(b, dim=1, keepdim=True) ** 2 / b.shape[1] + _EPS).sqrt()
    unit = b / rms
    sample = torch.arange(b.shape[0], device="cuda") // s["span"]
    gate = s["gate"].double()[sample]
    h = s["alpha"] * s["res"].double() + unit * s["post"].double() * gate
    return h, (torch.linalg.vector_norm(h, dim=1, keepdim=True) ** 2 / b.shape[1] + _EPS).sqrt(), unit, rms, gate, sample


def _exact_norm(case, s):
    h, rms_h, unit, rms_b, gate, sample = _exact_sum(case, s)
    pre, post, d = s["pre"].double(), s["post"].double(), h.shape[1]
    y = h / rms_h * pre
    if case["kind"] == "norm_serve":
        return {"h": h, "y": y}
    kept = h.to(s["b"].dtype).double() / rms_h
    dy = s["dy"].double()
    t = s["dh"].double() + (dy * pre - kept * (torch.einsum("nd,nd,d->n", dy, kept, pre) / d)[:, None]) / rms_h
    du = t * gate
    db = (du * post - unit * (torch.einsum("nd,nd,d->n", du, unit, post) / d)[:, None]) / rms_b
    dgate = torch.zeros(s["gate"].shape, dtype=torch.float64, device="cuda").index_add_(0, sample, t * unit * post)
    return {"h": h, "y": y, "db": db, "dres": s["alpha"] * t, "dgate": dgate, "dpost": torch.einsum("nd,nd->d", du, unit), "dpre": torch.einsum("nd,nd->d", dy, kept)}


def _exact_product_of(case, s, x, w):
    z = torch.empty((x.shape[0], w.shape[0]), dtype=torch.float64, device="cuda")
    bias = s["bias"].double() if s["bias"] is not None else torch.zeros(w.shape[0], dtype=torch.float64, device="cuda")
    for i in range(0, x.shape[0], 4096):
        torch.addmm(bias, x[i:i + 4096], w.t(), out=z[i:i + 4096])
    return z


def _exact_kept(q, scale, d):
    return q[:, :d].double() * scale.double()[:, None]


def _exact_linear_serve(case, s):
    h, rms, _, _, _, _ = _exact_sum(case, s)
    x, _ = _exact_rows(h / rms * s["pre"].double())
    return {"h": h, "z": _exact_product_of(case, s, x, _exact_kept(s["wq"], s["ws"], case["width"]))}


def _exact_product(case, s):
    return {"z": _exact_product_of(case, s, _exact_kept(s["xq"], s["xs"], case["width"]), _exact_kept(s["wq"], s["ws"], case["width"]))}


def _exact_checkpoint(case, s):
    x, scale = _exact_rows(s["x"].double())
    return {"x": x, "scale": scale}


def _exact_linear_train(case, s):
    (x, _), (w, _) = _exact_rows(s["x"].double()), _exact_rows(s["w"].double())
    dy, dt = s["dy"].double(), s["x"].dtype
    out = {"z": _exact_product_of(case, s, x, w)}
    # the gradients are those of the operands as they were kept, in the tensors' type
    x, w = x.to(dt).double(), w.to(dt).double()
    out |= {"dx": torch.einsum("no,od->nd", dy, w), "dw": torch.einsum("no,nd->od", dy, x)}
    if s["bias"] is not None:
        out["db"] = torch.einsum("no->o", dy)
    return out

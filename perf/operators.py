"""Measured cases of the operators at the tail of a language-model training step: dropout with the residual's
addition, RMS norm with the residual's addition (also to 8 bits), and the vocabulary projection with its softmax cross
entropy.  `own` chooses between the operators' plain forms (elementary torch operations in 32 bits) and the library's
kernels.

A case has a `kind`:
  ce_eval     loss of every row under the vocabulary projection (scoring)
  ce_train    loss and the gradients of rows, projection and bias
  norm_serve  residual addition + RMS norm to e4m3 values with one scale per `group` values (0: per row)
  norm_train  residual addition + RMS norm, and the backward pass
  dropout     dropout (+ residual addition) and its backward pass
"""
import math

import numpy as np
import torch

own = False

_DT = {"bf16": torch.bfloat16, "fp32": torch.float32}
_EPS = 1e-6
_E4M3_MAX = 448.0


def listed():
    return [
        # one position of one sequence is scored: latency, bound by reading the projection once
        _ce("ce_eval_one_row", "ce_eval", 1, 2048, 65536, "bf16"),
        # evaluation of a batch of sequences with sizes that fill no tile
        _ce("ce_eval_ragged", "ce_eval", 2001, 1000, 50021, "bf16"),
        # the classifier head of the CIFAR-100 networks at their batch size: smallest training call
        _ce("ce_train_head", "ce_train", 128, 64, 100, "bf16", bias=True),
        # training step of a small language model, a tenth of the rows padded
        _ce("ce_train_mid", "ce_train", 4096, 1024, 32000, "bf16", ignored=0.1),
        # the same in 32 bits, ragged in every size, with a bias
        _ce("ce_train_fp32", "ce_train", 1111, 520, 10007, "fp32", bias=True, ignored=0.1),
        # training step of a large language model on one GPU
        _ce("ce_train_large", "ce_train", 8192, 4096, 65536, "bf16"),
        # serving, one token
        _norm("norm_serve_one_row", "norm_serve", 1, 4096, "bf16", group=0),
        # serving, a prompt; one scale per 128 values
        _norm("norm_serve_prompt", "norm_serve", 4096, 8192, "bf16", group=128),
        # training at odd sizes in 32 bits
        _norm("norm_train_fp32", "norm_train", 777, 1021, "fp32"),
        # training, ordinary width
        _norm("norm_train", "norm_train", 8192, 4096, "bf16"),
        # hidden layer of the multilayer perceptron at batch 128
        _drop("dropout_small", 128 * 128, "fp32", False),
        # residual branch of a large training step
        _drop("dropout_large", 8192 * 4096, "bf16", True),
    ]


def _ce(name, kind, rows, width, vocab, dtype, bias=False, ignored=0.0):
    return {"name": name, "kind": kind, "rows": rows, "width": width, "vocab": vocab, "dtype": dtype, "bias": bias, "ignored": ignored}


def _norm(name, kind, rows, width, dtype, group=0):
    return {"name": name, "kind": kind, "rows": rows, "width": width, "dtype": dtype, "group": group}


def _drop(name, n, dtype, residual):
    return {"name": name, "kind": "dropout", "n": n, "dtype": dtype, "residual": residual, "p": 0.1}


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["ce_eval", "ce_train", "ce_train", "norm_serve", "norm_train", "dropout"])
    dtype = rng.choice(["bf16", "bf16", "bf16", "fp32"])
    if kind == "dropout":
        c = _drop("", _log(rng, 1000, 8192 * 4096), dtype, rng.random() < 0.5)
        c["p"] = rng.choice([0.05, 0.1, 0.25, 0.5])
    elif kind.startswith("norm"):
        rows, width = _log(rng, 1, 8192), _log(rng, 64, 8192)
        if rng.random() < 0.7:
            width = -(-width // 128) * 128
        while rows * width > 8192 * 4096:
            rows //= 2
        c = _norm("", kind, rows, width, "bf16" if kind == "norm_serve" else dtype, rng.choice([0, 128]) if width % 128 == 0 else 0)
    else:
        rows, width, vocab = _log(rng, 1, 8192), _log(rng, 64, 4096), _log(rng, 100, 65536)
        if rng.random() < 0.75:
            width = -(-width // 8) * 8
        # 32-bit products are worked in pieces of 16 bits: a quarter of the rows and of the vocabulary at most
        if dtype == "fp32":
            rows, vocab = min(rows, 2048), min(vocab, 16384)
        c = _ce("", kind, rows, width, vocab, dtype, rng.random() < 0.3, rng.choice([0.0, 0.1, 0.5]))
    del c["name"]
    return c


def _generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def prepare(case, seed):
    g, dt, kind = _generator(seed), _DT[case["dtype"]], case["kind"]

    def normal(*size, std=1.0, mean=0.0):
        return torch.empty(size, device="cuda", dtype=dt).normal_(mean, std, generator=g)

    s = {"case": case, "kind": kind}
    if kind == "dropout":
        s |= {"x": normal(case["n"]), "res": normal(case["n"]) if case["residual"] else None, "dy": normal(case["n"])}
        s["rng"] = torch.tensor([seed * 0x9E3779B97F4A7C15 % (1 << 62), seed * 1000003], dtype=torch.int64, device="cuda")
        return s
    n, d = case["rows"], case["width"]
    if kind.startswith("norm"):
        # a residual stream is wider than what a block adds to it; the weights of the norm are near one
        return s | {"x": normal(n, d), "res": normal(n, d, std=3.0), "gamma": normal(d, std=0.1, mean=1.0), "dy": normal(n, d), "dh": normal(n, d)}
    v = case["vocab"]
    # rows come out of a norm; the projection's scale gives logits of a few units
    s |= {"x": normal(n, d), "w": normal(v, d, std=2.0 / math.sqrt(d)), "bias": normal(v) if case["bias"] else None}
    labels = torch.randint(0, v, (n,), device="cuda", generator=g, dtype=torch.int32)
    if case["ignored"]:
        labels[torch.rand(n, device="cuda", generator=g) < case["ignored"]] = -1
    s["labels"] = labels
    return s


def run(state):
    kind = state["kind"]
    if own:
        return {"ce_eval": _own_ce_eval, "ce_train": _own_ce_train, "norm_serve": _own_norm_serve, "norm_train": _own_norm_train, "dropout": _own_dropout}[kind](state)
    return {"ce_eval": _ce_eval, "ce_train": _ce_train, "norm_serve": _norm_serve, "norm_train": _norm_train, "dropout": _dropout}[kind](state)


# ---- plain forms ---------------------------------------------------------------------------------------------------
def _logits(s):
    z = s["x"].float() @ s["w"].float().t()
    return z if s["bias"] is None else z + s["bias"].float()


def _losses(z, labels):
    top = z.amax(1, keepdim=True)
    lse = (z - top).exp().sum(1).log() + top[:, 0]
    counted = labels >= 0
    row = torch.where(counted, lse - z.gather(1, labels.clamp(min=0).long()[:, None])[:, 0], 0.0)
    count = counted.sum().clamp(min=1)
    return row, lse, row.sum() / count, counted, count


def _ce_eval(s):
    row, lse, loss, _, _ = _losses(_logits(s), s["labels"])
    return {"loss": loss, "row_loss": row, "lse": lse}


def _ce_train(s):
    z = _logits(s)
    _, lse, loss, counted, count = _losses(z, s["labels"])
    dz = (z - lse[:, None]).exp()
    dz.scatter_add_(1, s["labels"].clamp(min=0).long()[:, None], torch.full_like(lse, -1.0)[:, None])
    dz = torch.where(counted[:, None], dz / count, 0.0)
    dt = s["x"].dtype
    out = {"loss": loss, "dx": (dz @ s["w"].float()).to(dt), "dw": (dz.t() @ s["x"].float()).to(dt)}
    if s["bias"] is not None:
        out["db"] = dz.sum(0)
    return out


def _normed(s):
    h = s["x"].float() + s["res"].float()
    rstd = torch.rsqrt(h.square().mean(1) + _EPS)
    return h, rstd, h * rstd[:, None] * s["gamma"].float()


def _norm_serve(s):
    h, _, y = _normed(s)
    group = s["case"]["group"] or y.shape[1]
    blocks = y.view(y.shape[0], -1, group)
    top = blocks.abs().amax(2)
    scale = torch.where(top > 0, top / _E4M3_MAX, 1.0)
    return {"h": h.to(s["x"].dtype), "q": (blocks / scale[:, :, None]).view_as(y).to(torch.float8_e4m3fn), "scale": scale}


def _norm_train(s):
    dt = s["x"].dtype
    h, rstd, y = _normed(s)
    # the backward pass has the sum as it was stored
    kept, r = h.to(dt).float(), rstd[:, None]
    dy, gamma = s["dy"].float(), s["gamma"].float()
    wdy = dy * gamma
    dx = s["dh"].float() + r * (wdy - kept * (r * r) * (wdy * kept).mean(1, keepdim=True))
    return {"h": h.to(dt), "y": y.to(dt), "rstd": rstd, "dx": dx.to(dt), "dgamma": (dy * kept * r).sum(0)}


def _philox(rng, count, layer):
    """Philox4x32-10 (Salmon et al., 2011): `count` blocks of four 32-bit words from the 64-bit counters that start at
    rng[1] (low words of the counter; the third word is the layer), under the 64-bit key rng[0]."""
    low = 0xFFFFFFFF
    at = rng[1] + torch.arange(count, device=rng.device)
    a, b, c, d = at & low, (at >> 32) & low, torch.full_like(at, layer), torch.zeros_like(at)
    k0, k1 = rng[0] & low, (rng[0] >> 32) & low
    for _ in range(10):
        p, q = a * 0xD2511F53, c * 0xCD9E8D57
        a, b, c, d = ((q >> 32) & low) ^ b ^ k0, q & low, ((p >> 32) & low) ^ d ^ k1, p & low
        k0, k1 = (k0 + 0x9E3779B9) & low, (k1 + 0xBB67AE85) & low
    return torch.stack([a, b, c, d], 1)


def _dropout(s):
    x, n, dt = s["x"], s["case"]["n"], s["x"].dtype
    t = round(s["case"]["p"] * 65536)
    words = _philox(s["rng"], -(-n // 8), 0)
    keep = torch.stack([words & 0xFFFF, words >> 16], 2).reshape(-1)[:n] >= t
    scale = 65536.0 / (65536 - t)
    y = torch.where(keep, x.float() * scale, 0.0)
    if s["res"] is not None:
        y = y + s["res"].float()
    return {"y": y.to(dt), "dx": torch.where(keep, s["dy"].float() * scale, 0.0).to(dt)}


# ---- the library's kernels -----------------------------------------------------------------------------------------
def _prec(t):
    return 1 if t.dtype == torch.bfloat16 else 0


def _f32(*size):
    return torch.empty(size, dtype=torch.float32, device="cuda")


def _own_ce_fwd(s, ws, stream):
    from paper_1804_10574_b200 import binding
    x, w = s["x"], s["w"]
    (n, d), v = x.shape, w.shape[0]
    loss, row, lse = _f32(1), _f32(n), _f32(n)
    binding.linear_ce_fwd(_prec(x), x, w, s["bias"], s["labels"], loss, row, lse, ws, n, d, v, stream)
    return loss, row, lse


def _workspace(s, backward):
    from paper_1804_10574_b200 import binding
    x, w = s["x"], s["w"]
    return torch.empty(binding.linear_ce_workspace_bytes(_prec(x), x.shape[0], x.shape[1], w.shape[0], backward), dtype=torch.uint8, device="cuda")


def _own_ce_eval(s):
    loss, row, lse = _own_ce_fwd(s, _workspace(s, False), torch.cuda.current_stream().cuda_stream)
    return {"loss": loss[0], "row_loss": row, "lse": lse}


def _own_ce_train(s):
    from paper_1804_10574_b200 import binding
    x, w, stream = s["x"], s["w"], torch.cuda.current_stream().cuda_stream
    ws = _workspace(s, True)
    loss, _, lse = _own_ce_fwd(s, ws, stream)
    dx, dw = torch.empty_like(x), torch.empty_like(w)
    db = _f32(w.shape[0]) if s["bias"] is not None else None
    binding.linear_ce_bwd(_prec(x), x, w, s["bias"], s["labels"], lse, None, None, dx, dw, db, ws, x.shape[0], x.shape[1], w.shape[0], False, stream)
    out = {"loss": loss[0], "dx": dx, "dw": dw}
    if db is not None:
        out["db"] = db
    return out


def _own_norm_serve(s):
    from paper_1804_10574_b200 import binding
    x, group = s["x"], s["case"]["group"]
    n, d = x.shape
    h, q, scale = torch.empty_like(x), torch.empty((n, d), dtype=torch.float8_e4m3fn, device="cuda"), _f32(n, d // (group or d))
    binding.add_rmsnorm_fwd(_prec(x), x, s["res"], s["gamma"], h, None, q, scale, None, n, d, group, _EPS, torch.cuda.current_stream().cuda_stream)
    return {"h": h, "q": q, "scale": scale}


def _own_norm_train(s):
    from paper_1804_10574_b200 import binding
    x, stream = s["x"], torch.cuda.current_stream().cuda_stream
    n, d = x.shape
    h, y, rstd, dx, dgamma = torch.empty_like(x), torch.empty_like(x), _f32(n), torch.empty_like(x), _f32(d)
    binding.add_rmsnorm_fwd(_prec(x), x, s["res"], s["gamma"], h, y, None, None, rstd, n, d, 0, _EPS, stream)
    scratch = _f32(binding.rmsnorm_scratch_elems(n, d))
    binding.add_rmsnorm_bwd(_prec(x), s["dy"], s["dh"], h, s["gamma"], rstd, dx, dgamma, scratch, n, d, stream)
    return {"h": h, "y": y, "rstd": rstd, "dx": dx, "dgamma": dgamma}


def _own_dropout(s):
    from paper_1804_10574_b200 import binding
    x, n, p, stream = s["x"], s["case"]["n"], s["case"]["p"], torch.cuda.current_stream().cuda_stream
    y, dx = torch.empty_like(x), torch.empty_like(x)
    binding.dropout_fwd(_prec(x), x, s["res"], y, s["rng"], n, p, 0, stream)
    binding.dropout_bwd(_prec(x), s["dy"], dx, s["rng"], n, p, 0, stream)
    return {"y": y, "dx": dx}


# ---- work ----------------------------------------------------------------------------------------------------------
def work(case):
    e = 2 if case["dtype"] == "bf16" else 4
    if case["kind"] == "dropout":
        n = case["n"]
        return {"bytes": n * e * (4 + (1 if case["residual"] else 0)), "flops": 4 * n}
    n, d = case["rows"], case["width"]
    if case["kind"] == "norm_serve":
        return {"bytes": n * d * (3 * e + 1) + d * e + 4 * n * (d // (case["group"] or d)), "flops": 6 * n * d}
    if case["kind"] == "norm_train":
        # forward x, res -> h, y; backward dy, dh, h -> dx (the sum is read again after all rows were written)
        return {"bytes": 8 * n * d * e + 8 * n + d * (2 * e + 4), "flops": 18 * n * d}
    v = case["vocab"]
    flops, moved = 2 * n * v * d, (n + v) * d * e + 12 * n + (v * e if case["bias"] else 0)
    if case["kind"] == "ce_train":
        # the two products of the backward pass; the logits' second computation is the price of not keeping them
        flops, moved = 3 * flops, moved + (n + v) * d * e + (4 * v if case["bias"] else 0)
    return {"bytes": moved, "flops": flops}


# ---- 64 bits -------------------------------------------------------------------------------------------------------
def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] == "dropout":
        return _exact_dropout(case, s)
    if case["kind"].startswith("norm"):
        return _exact_norm(case, s)
    return _exact_ce(case, s)


def _exact_dropout(case, s):
    n, t = case["n"], int(case["p"] * 65536 + 0.5)
    key, start = (int(v) for v in s["rng"].tolist())
    m32, sh = np.uint64(0xFFFFFFFF), np.uint64(32)
    at = np.arange((n + 7) // 8, dtype=np.uint64) + np.uint64(start)
    ctr = [at & m32, at >> sh, np.zeros_like(at), np.zeros_like(at)]
    k = [key % (1 << 32), key >> 32]
    for r in range(10):
        lo, hi = ctr[0] * np.uint64(0xD2511F53), ctr[2] * np.uint64(0xCD9E8D57)
        ctr = [(hi >> sh) ^ ctr[1] ^ np.uint64(k[0]), hi & m32, (lo >> sh) ^ ctr[3] ^ np.uint64(k[1]), lo & m32]
        k = [(k[0] + 0x9E3779B9) % (1 << 32), (k[1] + 0xBB67AE85) % (1 << 32)]
    u = np.empty((len(at), 8), dtype=np.uint16)
    for j in range(4):
        u[:, 2 * j], u[:, 2 * j + 1] = ctr[j] & np.uint64(0xFFFF), ctr[j] >> np.uint64(16)
    keep = u.reshape(-1)[:n] >= t
    scale = 65536 / (65536 - t)
    f64 = lambda v: v.double().cpu().numpy()  # noqa: E731
    y = np.where(keep, f64(s["x"]) * scale, 0.0) + (f64(s["res"]) if s["res"] is not None else 0.0)
    return {"y": y, "dx": np.where(keep, f64(s["dy"]) * scale, 0.0)}


def _exact_norm(case, s):
    x, res, gamma = s["x"].double(), s["res"].double(), s["gamma"].double()
    n, d = x.shape
    h = x + res
    rms = (torch.linalg.vector_norm(h, dim=1) ** 2 / d + _EPS).sqrt()
    unit = h / rms[:, None]
    y = unit * gamma
    if case["kind"] == "norm_serve":
        parts = y.reshape(n, -1, case["group"] or d)
        scale = torch.linalg.vector_norm(parts, ord=math.inf, dim=2) / _E4M3_MAX
        return {"h": h, "q": (parts / scale[..., None]).reshape(n, d), "scale": scale}
    # the backward pass is that of the stored sum
    kept = h.to(s["x"].dtype).double() / rms[:, None]
    dy = s["dy"].double()
    dot = torch.einsum("nd,nd,d->n", dy, kept, gamma) / d
    return {"h": h, "y": y, "rstd": 1 / rms, "dx": s["dh"].double() + (dy * gamma - kept * dot[:, None]) / rms[:, None], "dgamma": torch.einsum("nd,nd->d", dy, kept)}


def _exact_ce(case, s):
    x, w, labels = s["x"].double(), s["w"].double(), s["labels"].long()
    n, v = x.shape[0], w.shape[0]
    bias = s["bias"].double() if s["bias"] is not None else torch.zeros(v, dtype=torch.float64, device="cuda")
    counted = (labels >= 0).double()
    count = max(1.0, float(counted.sum()))
    train = case["kind"] == "ce_train"
    row, lse = torch.zeros_like(x[:, 0]), torch.zeros_like(x[:, 0])
    dx, dw, db = torch.zeros_like(x), torch.zeros_like(w) if train else None, torch.zeros_like(bias)
    for i in range(0, n, 2048):
        part = slice(i, i + 2048)
        z = torch.addmm(bias, x[part], w.t())
        lse[part] = torch.logsumexp(z, 1)
        hit = torch.nn.functional.one_hot(labels[part].clamp(min=0), v).double()
        row[part] = (lse[part] - (z * hit).sum(1)) * counted[part]
        if train:
            dz = (torch.softmax(z, 1) - hit) * (counted[part] / count)[:, None]
            dx[part] = dz @ w
            dw.addmm_(dz.t(), x[part])
            db += dz.sum(0)
    loss = row.sum() / count
    if not train:
        return {"loss": loss, "row_loss": row, "lse": lse}
    out = {"loss": loss, "dx": dx, "dw": dw}
    if s["bias"] is not None:
        out["db"] = db
    return out

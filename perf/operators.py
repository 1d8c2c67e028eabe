"""The 8-bit operators around the block's products, and how they are used.

One format joins them: int8 codes q in [-127, 127] with an fp32 scale per row
(a row's values are scale * q).  The code of z in a row whose largest
magnitude is A is the integer nearest to 127 z / A, ties to even.

    norm       h = x + residual, y = RMSNorm(h) w          (bf16 output)
    norm_int8  the same with the output as codes and scales, one per token
    norm_back  the norm's backward: input and weight gradient
    product    C = (a sa) (b sb)^T + residual from codes and scales, one per
               token and one per output channel
    serve      norm_int8, then product: one layer's input projection
    save       activations to codes, and back to bf16
    back       a linear layer's weight gradient from its saved 8-bit input

    listed()                 the named cases
    draw(rng)                one more case of the same ranges
    prepare(case, seed)      what the program holds before the call
    run(state)               one pass; returns every output whole
    work(case)               bytes and flops that the pass cannot do without
    exact(case, seed)        the same outputs in 64 bits

`own` says whether run() calls this package or computes the plain form.
"""
from __future__ import annotations

import math

import torch

own = False

EPS = 1e-5
DEVICE = "cuda"


def listed():
    return [
        # generation of one sequence: one token enters a layer; latency alone
        dict(kind="norm", rows=1, d=2048, residual=True, name="norm_one"),
        # the norm of a 65,536-token training step of the 1B model
        dict(kind="norm", rows=65536, d=2048, residual=True, name="norm_step"),
        # a ragged prompt batch of a small model, codes for an int8 product
        dict(kind="norm_int8", rows=4999, d=1416, residual=True, name="norm_int8_ragged"),
        # backward of a small model's step
        dict(kind="norm_back", rows=2048, d=1024, residual=False, name="norm_back_small"),
        # backward of the 65,536-token step, the residual path's gradient added
        dict(kind="norm_back", rows=65536, d=2048, residual=True, name="norm_back_step"),
        # one token through the norm and the query/key/value projection
        dict(kind="serve", rows=1, d=2048, n=6144, residual=True, name="serve_one"),
        # the logits of 16 sequences that generate together, 50,432-token
        # vocabulary: the weights' bytes
        dict(kind="product", rows=16, d=2048, n=50432, residual=False, name="product_head"),
        # a prompt batch whose sizes no tile divides
        dict(kind="product", rows=1531, d=1040, n=5001, residual=True, name="product_ragged"),
        # the MLP's input projection of the whole step: matrix-core bound
        dict(kind="product", rows=65536, d=2048, n=5632, residual=False, name="product_step"),
        # the gate product of a quarter step saved and restored
        dict(kind="save", rows=16384, d=5632, wide=False, name="save_gate"),
        # weight gradient of a ragged batch of a small model
        dict(kind="back", rows=3001, d=1040, n=1416, name="back_ragged"),
        # weight gradient of the MLP's input projection over the whole step
        dict(kind="back", rows=65536, d=2048, n=5632, name="back_step"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["norm", "norm_int8", "norm_back", "serve", "product", "product", "save",
                       "back", "back"])
    rows = _log_int(rng, 1, 65536)
    if kind in ("norm", "norm_int8", "norm_back", "save"):
        d = _log_int(rng, 64, 8192)
        if rng.random() < 0.75:  # aligned rows; the others are of any length
            d = max(64, d // 8 * 8)
        rows = max(1, min(rows, 65536 * 2048 // d))
        if kind == "save":
            return dict(kind=kind, rows=rows, d=d, wide=rng.random() < 0.3)
        return dict(kind=kind, rows=rows, d=d, residual=rng.random() < 0.6)
    d, n = 16 * _log_int(rng, 4, 384), _log_int(rng, 64, 8192)
    if kind == "back":
        n = max(64, n // 8 * 8)
    rows = max(1, min(rows, 65536 * 2048 * 5632 // (d * n), 65536 * 2048 // d, 65536 * 5632 // n))
    case = dict(kind=kind, rows=rows, d=d, n=n)
    if kind != "back":
        case["residual"] = rng.random() < 0.5
    return case


# ---------------------------------------------------------------------------
# inputs


def _bf16(x):
    return x.to(torch.bfloat16)


def _normal(gen, *shape):
    return torch.randn(shape, generator=gen, device=DEVICE, dtype=torch.float32)


def _activations(gen, rows, d):
    """Activations: channels of different size, and a few outliers among them."""
    gain = torch.exp(0.4 * _normal(gen, d))
    gain[torch.rand(d, generator=gen, device=DEVICE) < 0.01] *= 8
    return _bf16(_normal(gen, rows, d).mul_(gain))


def _inputs(case, seed):
    """The tensors of a pass, by name, from the seed alone."""
    gen = torch.Generator(device=DEVICE).manual_seed(int(seed))
    kind, rows, d = case["kind"], case["rows"], case["d"]
    if kind == "save":
        if case["wide"]:  # the middle columns of a wider matrix
            return {"x": _activations(gen, rows, d + 64)[:, 32:32 + d]}
        return {"x": _activations(gen, rows, d)}
    t = {}
    if kind in ("norm", "norm_int8", "norm_back", "serve"):
        t["w"] = _bf16(1 + 0.1 * _normal(gen, d))
    if kind in ("norm", "norm_int8", "serve", "back"):
        t["x"] = _activations(gen, rows, d)
    if kind in ("norm", "norm_int8", "serve"):
        t["residual"] = _activations(gen, rows, d) if case["residual"] else None
    if kind == "norm_back":
        t["h"], t["dy"] = _activations(gen, rows, d), _bf16(_normal(gen, rows, d))
        t["rstd"] = _rstd(t["h"].float())
        t["dres"] = _bf16(_normal(gen, rows, d)) if case["residual"] else None
    if kind == "back":
        t["dy"] = _bf16(_normal(gen, rows, case["n"]))
    if kind in ("serve", "product"):
        t["b"], t["sb"] = _codes(_bf16(0.02 * _normal(gen, case["n"], d)))
    if kind == "product":
        t["a"], t["sa"] = _codes(_activations(gen, rows, d))
        t["residual"] = _bf16(_normal(gen, rows, case["n"])) if case["residual"] else None
    return t


def prepare(case, seed):
    return dict(case=case, t=_inputs(case, seed))


# ---------------------------------------------------------------------------
# the plain form


def _rstd(h):
    return 1 / torch.sqrt(h.square().mean(1) + EPS)


def _scaled_codes(z, amax):
    """The nearest integers to 127 z / amax (fp32 tensors), ties to even.  In
    64 bits: 127 z has 23 significant bits, so the quotient is on the right
    side of every border, and on it where z is."""
    q = torch.round(z.double().mul_(127).div_(amax.double()[:, None]))
    return q.nan_to_num_(0.0).to(torch.int8)  # 0 / 0: a row of zeros


def _codes(x):
    x = x.float()
    amax = x.abs().amax(1)
    return _scaled_codes(x, amax), amax / 127


def _norm_codes(h, rstd, w):
    z = h * w.float()  # exact: 8 significant bits each
    amax = z.abs().amax(1)
    return _scaled_codes(z, amax), amax * rstd / 127


def _sum(x, residual):
    return x if residual is None else _bf16(x.float() + residual.float())


def _values(q, s):
    return _bf16(q.float() * s[:, None])


def _product(a, sa, b, sb, residual):
    c = torch.matmul(a.float(), b.float().t()) * sa[:, None] * sb
    return _bf16(c if residual is None else c + residual.float())


def _plain(case, t):
    kind = case["kind"]
    if kind == "norm":
        h = _sum(t["x"], t["residual"])
        rstd = _rstd(h.float())
        y = _bf16(h.float() * rstd[:, None] * t["w"].float())
        return {"y": y, "h": h, "rstd": rstd}
    if kind == "norm_int8":
        h = _sum(t["x"], t["residual"])
        rstd = _rstd(h.float())
        q, s = _norm_codes(h.float(), rstd, t["w"])
        return {"y": _values(q, s), "scales": s, "h": h, "rstd": rstd}
    if kind == "norm_back":
        xh = t["h"].float() * t["rstd"][:, None]
        dy = t["dy"].float()
        g = dy * t["w"].float()
        dx = (g - xh * (g * xh).mean(1, keepdim=True)) * t["rstd"][:, None]
        if t["dres"] is not None:
            dx = dx + t["dres"].float()
        return {"dx": _bf16(dx), "dw": _bf16((dy * xh).sum(0))}
    if kind == "serve":
        h = _sum(t["x"], t["residual"])
        q, s = _norm_codes(h.float(), _rstd(h.float()), t["w"])
        return {"h": h, "c": _product(q, s, t["b"], t["sb"], None)}
    if kind == "product":
        return {"c": _product(t["a"], t["sa"], t["b"], t["sb"], t["residual"])}
    q, s = _codes(t["x"])
    if kind == "save":
        return {"x": _values(q, s), "scales": s}
    # the restored activations are bf16, as the ones that were saved
    return {"dw": _bf16(torch.matmul(_values(q, s).float().t(), t["dy"].float())), "scales": s}


def _kernels(case, t):
    from paper_2405_13226_amd import block_ops as ops
    kind = case["kind"]
    if kind == "norm":
        y, h, rstd = ops.rms_norm(t["x"], t["w"], residual=t["residual"], eps=EPS)
        return {"y": y, "h": h, "rstd": rstd}
    if kind == "norm_int8":
        q, s, h, rstd = ops.rms_norm_int8(t["x"], t["w"], residual=t["residual"], eps=EPS)
        return {"y": ops.dequantize(q, s), "scales": s, "h": h, "rstd": rstd}
    if kind == "norm_back":
        dx, dw = ops.rms_norm_backward(t["h"], t["w"], t["rstd"], t["dy"], dres=t["dres"])
        return {"dx": dx, "dw": dw}
    if kind == "serve":
        q, s, h, _ = ops.rms_norm_int8(t["x"], t["w"], residual=t["residual"], eps=EPS)
        return {"h": h, "c": ops.gemm_int8(q, s, t["b"], t["sb"])}
    if kind == "product":
        return {"c": ops.gemm_int8(t["a"], t["sa"], t["b"], t["sb"], residual=t["residual"])}
    q, s = ops.quantize(t["x"])
    if kind == "save":
        return {"x": ops.dequantize(q, s), "scales": s}
    return {"dw": ops.gemm_int8_wgrad(q, s, t["dy"]), "scales": s}


def run(state):
    if own:
        return _kernels(state["case"], state["t"])
    return _plain(state["case"], state["t"])


# ---------------------------------------------------------------------------
# what a pass cannot do without


def work(case):
    kind, rows, d = case["kind"], case["rows"], case["d"]
    res = 1 if case.get("residual") else 0
    if kind in ("norm", "norm_int8"):
        # x, residual, weight in; y, h (x itself without a residual), rstd
        # and scales out
        stats = 4 if kind == "norm" else 8
        return dict(bytes=2 * rows * d * (2 + 2 * res) + 2 * d + stats * rows, flops=4 * rows * d)
    if kind == "norm_back":
        return dict(bytes=2 * rows * d * (3 + res) + 4 * d + 4 * rows, flops=10 * rows * d)
    if kind == "save":
        return dict(bytes=4 * rows * d + 4 * rows, flops=2 * rows * d)
    n = case["n"]
    if kind == "serve":
        return dict(bytes=2 * rows * d * (1 + 2 * res) + 2 * d + n * d + 4 * n + 2 * rows * n,
                    flops=2 * rows * n * d)
    if kind == "product":
        return dict(bytes=rows * d + 4 * rows + n * d + 4 * n + 2 * rows * n * (1 + res),
                    flops=2 * rows * n * d)
    return dict(bytes=2 * rows * (d + n) + 2 * d * n + 4 * rows, flops=2 * rows * n * d)


# ---------------------------------------------------------------------------
# the same outputs in 64 bits, from the definitions


def exact(case, seed):
    t = _inputs(case, seed)
    f = {k: v.double() for k, v in t.items() if v is not None}
    kind = case["kind"]

    def nearest(z):
        """(codes, largest magnitude) of the rows of z."""
        top = z.abs().max(dim=1, keepdim=True).values
        return torch.where(top > 0, torch.round(127 * z / top), 0 * z), top

    if kind in ("norm", "norm_int8", "serve"):
        h = f["x"]
        if "residual" in f:  # the stream is kept in bf16
            h = (h + f["residual"]).to(torch.bfloat16).double()
        rstd = (h.pow(2).sum(dim=1) / case["d"] + EPS) ** -0.5
        if kind == "norm":
            return {"y": h * rstd[:, None] * f["w"], "h": h, "rstd": rstd}
        q, top = nearest(h * f["w"])
        scales = top[:, 0] * rstd / 127
        if kind == "norm_int8":
            return {"y": q * scales[:, None], "scales": scales, "h": h, "rstd": rstd}
        return {"h": h, "c": (q @ f["b"].t()) * torch.outer(scales, f["sb"])}
    if kind == "norm_back":
        h, dy, r = f["h"], f["dy"], f["rstd"][:, None]
        inner = (dy * f["w"] * h).sum(dim=1, keepdim=True) / case["d"]
        dx = dy * f["w"] * r - h * inner * r ** 3
        return {"dx": dx + f["dres"] if "dres" in f else dx, "dw": (dy * h * r).sum(dim=0)}
    if kind == "product":
        c = (f["a"] @ f["b"].t()) * torch.outer(f["sa"], f["sb"])
        return {"c": c + f["residual"] if "residual" in f else c}
    q, top = nearest(f["x"])
    if kind == "save":
        return {"x": q * top / 127, "scales": top[:, 0] / 127}
    restored = (q * top / 127).to(torch.bfloat16).double()  # kept in bf16
    return {"dw": restored.t() @ f["dy"], "scales": top[:, 0] / 127}

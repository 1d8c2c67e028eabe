"""The 8-bit operators in float64 numpy, from their definitions."""
import numpy as np
import torch


def bf16(shape, seed, scale=1.0):
    g = torch.Generator(device="cpu").manual_seed(seed)
    return (torch.randn(shape, generator=g) * scale).to(torch.bfloat16)


def f64(t):
    return t.float().cpu().numpy().astype(np.float64)


def round_bf16(x):
    """Float64 values that bf16 or fp32 arithmetic gave, rounded to bf16."""
    return torch.from_numpy(np.asarray(x)).to(torch.float32).to(torch.bfloat16)


def codes(z):
    """(codes, largest magnitude) per row: the integers nearest to 127 z / A,
    ties to even.  127 z is exact in float64, and a quotient of two numbers of
    at most 23 significant bits is never rounded onto a border it is not on."""
    top = np.abs(z).max(1)
    with np.errstate(invalid="ignore", divide="ignore"):
        q = np.rint(127.0 * z / top[:, None])
    bad = ~np.isfinite(top) | (top == 0)
    q[bad] = 0
    return q.astype(np.int8), top


def add(x, r):
    """bf16(x + r) as the norm forms it (fp32 sum, one rounding)."""
    return (x.float() + r.float()).to(torch.bfloat16)


def rstd(h, eps):
    return 1.0 / np.sqrt((h * h).mean(1) + eps)


def norm_backward(h, w, rs, dy, dres=None):
    """(dx, dw, the magnitude that dx's fp32 rounding errors scale with)."""
    xh, g = h * rs[:, None], dy * w
    dx = rs[:, None] * (g - xh * (g * xh).mean(1, keepdims=True))
    mag = rs[:, None] * (np.abs(g) + np.abs(xh) * np.abs(g * xh).mean(1, keepdims=True))
    if dres is not None:
        dx, mag = dx + dres, mag + np.abs(dres)
    return dx, (dy * xh).sum(0), mag


def product(a, sa, b, sb):
    return (a.astype(np.float64) @ b.astype(np.float64).T) * np.outer(sa, sb)

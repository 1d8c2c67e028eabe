"""Log probabilities of given tokens from a model's logits, with the entropy
and the most likely alternatives, and their gradient: what a loss is made of
and what a text is scored with.

Argument marshalling only, as in ``attention.py``; the kernels are behind
dd_logprobs_fwd and dd_logprobs_bwd of include/dd_attn.h.

Logits are [rows, V] in bf16 or fp32 with unit column stride (the columns of a
wider, padded matrix are fine), targets int64 [rows]; a negative target is
ignored, one of V or more makes its log probability and that one's gradient NaN.
Statistics are fp32.
"""
from __future__ import annotations

import torch
from torch.autograd.function import once_differentiable

from .attention import _ptr as _p
from .block_ops import _call, _vec
from .cache import _F32, _bytes, _is

MAX_TOP = 64
_TYPES = (torch.bfloat16, torch.float32)


def _logits(t, name, dev=None):
    """(rows, V, row stride, whether fp32)."""
    if isinstance(t, torch.Tensor) and t.dim() == 2:
        (rows, V), (ld, one) = t.shape, t.stride()
        if (V and (one == 1 or V == 1) and t.is_cuda and t.dtype in _TYPES
                and (dev is None or t.device == dev)):
            return rows, V, ld if rows > 1 else V, t.dtype is torch.float32
    if not isinstance(t, torch.Tensor) or t.dim() != 2:
        raise ValueError(f"{name} must be a 2-D tensor")
    if t.dtype not in _TYPES or not t.is_cuda:
        raise ValueError(f"{name} must be a bf16 or fp32 GPU tensor")
    if dev is not None and t.device != dev:
        raise ValueError(f"{name} is on {t.device}, not on {dev}")
    if not t.shape[1]:
        raise ValueError(f"the rows of {name} are empty")
    raise ValueError(f"{name} must have unit column stride")


def logprobs(logits, targets, top: int = 0):
    """(logp, entropy, lse) of each row, fp32: the target's log probability, the
    entropy, and the log of the sum of exponentials; with ``top`` also the log
    probabilities (fp32 [rows, top]) and ids (int64) of the most likely tokens,
    in order, equal ones by the lowest id."""
    return _logprobs(logits, targets, top, True)


def _logprobs(logits, targets, top, shared):
    """shared: logp, entropy and lse are rows of one tensor (one allocation)."""
    rows, V, ldx, f32 = _logits(logits, "logits")
    dev = logits.device
    _vec(targets, "targets", rows, torch.int64, dev)
    if not 0 <= top <= min(V, MAX_TOP):
        raise ValueError(f"top must be at most {min(V, MAX_TOP)} (got {top})")
    if shared:
        logp, entropy, lse = logits.new_empty((3, rows), dtype=_F32).unbind()
    else:
        logp, entropy, lse = (logits.new_empty(rows, dtype=_F32) for _ in range(3))
    best = ids = None
    if top:
        best = logits.new_empty((rows, top), dtype=_F32)
        ids = targets.new_empty((rows, top))
    if rows:
        need = _bytes("dd_logprobs_workspace_bytes", rows, V, top)
        ws = torch.empty(need, dtype=torch.uint8, device=dev) if need else None
        _call(dev, "dd_logprobs_fwd", logits.data_ptr(), ldx, f32, targets.data_ptr(),
              logp.data_ptr(), entropy.data_ptr(), lse.data_ptr(), _p(best), _p(ids), rows, V, top,
              _p(ws), need)
    return (logp, entropy, lse, best, ids) if top else (logp, entropy, lse)


def logprobs_backward(logits, targets, lse, entropy, g_logp=None, g_entropy=None, g_lse=None,
                      out=None):
    """The gradient of the logits for the gradients of ``logprobs``' results
    (fp32 [rows], each optional), of their type; ``out`` (optional) receives it
    and may be the logits themselves."""
    rows, V, ldx, f32 = _logits(logits, "logits")
    dev, i = logits.device, logits.get_device()
    try:
        n = (rows,)
        fine = (_is(targets, n, torch.int64, i) and _is(lse, n, _F32, i) and _is(entropy, n, _F32, i)
                and (g_logp is None or _is(g_logp, n, _F32, i))
                and (g_entropy is None or _is(g_entropy, n, _F32, i))
                and (g_lse is None or _is(g_lse, n, _F32, i)))
    except AttributeError:
        fine = False
    if not fine:
        _vec(targets, "targets", rows, torch.int64, dev)
        for t, name in ((lse, "lse"), (entropy, "entropy"), (g_logp, "g_logp"),
                        (g_entropy, "g_entropy"), (g_lse, "g_lse")):
            if t is not None or name in ("lse", "entropy"):
                _vec(t, name, rows, torch.float32, dev)
    ldd = V
    if out is None:
        out = torch.empty_like(logits) if ldx == V else logits.new_empty((rows, V))
    else:
        r, c, ldd, same = _logits(out, "out", dev)
        if (r, c, same) != (rows, V, f32):
            raise ValueError(f"out must be a {logits.dtype} tensor of shape {(rows, V)}")
    if rows:
        _call(dev, "dd_logprobs_bwd", logits.data_ptr(), ldx, f32, targets.data_ptr(),
              lse.data_ptr(), entropy.data_ptr(), _p(g_logp), _p(g_entropy), _p(g_lse),
              out.data_ptr(), ldd, rows, V)
    return out


class LogProbFunction(torch.autograd.Function):
    """Autograd wrapper: the forward keeps the logits and each row's lse and
    entropy; alternatives carry no gradient."""

    @staticmethod
    def forward(ctx, logits, targets, top):
        res = _logprobs(logits, targets, top, False)
        ctx.save_for_backward(logits, targets, res[2], res[1])
        ctx.set_materialize_grads(False)
        ctx.mark_non_differentiable(*res[3:])
        return res

    @staticmethod
    @once_differentiable
    def backward(ctx, g_logp, g_entropy, g_lse, *_):
        logits, targets, lse, entropy = ctx.saved_tensors
        if g_logp is None and g_entropy is None and g_lse is None:
            return None, None, None
        grads = [None if g is None else g.contiguous() for g in (g_logp, g_entropy, g_lse)]
        return logprobs_backward(logits, targets, lse, entropy, *grads), None, None


def token_logprobs(logits, targets, top: int = 0):
    """Differentiable ``logprobs`` (in the logits, through logp, entropy and
    lse).  A training loss with a z term:

        logp, _, lse = token_logprobs(logits, targets)
        loss = -logp.mean() + 1e-4 * lse.square().mean()

    Where a captured graph shall hold the backward pass while eager autograd
    graphs of the same leaves live, capture ``logprobs`` and
    ``logprobs_backward``: autograd would join the two graphs' streams.
    """
    return LogProbFunction.apply(logits, targets, top)

"""Python binding of the block kernels around the attention (argument
marshalling only): the bf16 GEMM, LayerNorm and SwiGLU of include/dd_attn.h,
and its 8-bit operators: RMSNorm, rows as codes, and their products.

Every computation runs in the HIP kernels behind the C ABI; this module
checks tensor metadata, allocates outputs and scratch with torch on the
tensors' device and passes raw pointers, strides and the current stream.
Matrices are 2-D bf16 tensors with unit column stride (row-major, possibly
a column slice of a wider matrix: the row stride is passed through).

8-bit matrices are int8 codes [rows, d] with one fp32 scale per row: row r's
values are scales[r] * codes[r].  ``quantize`` forms them (the nearest codes
to 127 x / max |x| of each row, ties to even) and so does ``rms_norm_int8``;
``gemm_int8`` multiplies two of them, ``gemm_int8_wgrad`` takes one as the
kept input of a linear layer.  Their calls run on the tensors' device, on
its current stream; matrices without rows give empty results.  Rows have at
most 16384 elements (products: see there).
"""
from __future__ import annotations

import ctypes
import functools

import torch

from ._lib import check, lib
from .attention import _ptr as _p, _stream

LN_EPS = 1e-5
MAX_ROW = 16384  # elements of a row that RMSNorm takes or that is held as codes


def _mat(t, name):
    if (isinstance(t, torch.Tensor) and t.dim() == 2 and t.is_cuda
            and t.dtype is torch.bfloat16 and t.stride(1) == 1):
        return
    if not isinstance(t, torch.Tensor) or t.dim() != 2:
        raise ValueError(f"{name} must be a 2-D tensor")
    if t.device.type != "cuda" or t.dtype != torch.bfloat16:
        raise ValueError(f"{name} must be a bf16 GPU tensor")
    if t.stride(1) != 1:
        raise ValueError(f"{name} must have unit column stride")


def gemm(a, b, trans_a: bool = False, trans_b: bool = False, residual=None, out=None):
    """op(a) @ op(b) (+ residual) in bf16 with fp32 accumulation.

    op(a) = a, or a.T when ``trans_a`` (a stored [K, M]); op(b) likewise.
    ``out`` (optional) receives the result and may be ``residual`` itself."""
    _mat(a, "a")
    _mat(b, "b")
    M, K = (a.shape[1], a.shape[0]) if trans_a else (a.shape[0], a.shape[1])
    Kb, N = (b.shape[1], b.shape[0]) if trans_b else (b.shape[0], b.shape[1])
    if K != Kb:
        raise ValueError(f"inner dimensions differ: {K} vs {Kb}")
    if out is None:
        out = torch.empty((M, N), dtype=torch.bfloat16, device=a.device)
    _mat(out, "out")
    if tuple(out.shape) != (M, N):
        raise ValueError(f"out has shape {tuple(out.shape)}, expected {(M, N)}")
    if residual is not None:
        _mat(residual, "residual")
        if tuple(residual.shape) != (M, N) or residual.stride(0) != out.stride(0):
            raise ValueError("residual must match out in shape and row stride")
    need = lib().dd_gemm_workspace_bytes(M, N, K)
    ws = torch.empty(max(need, 1), dtype=torch.uint8, device=a.device) if need else None
    st = lib().dd_gemm(_p(a), a.stride(0), int(bool(trans_a)), _p(b), b.stride(0),
                       int(bool(trans_b)), _p(residual), _p(out), out.stride(0), M, N, K,
                       _p(ws), need, _stream(a.device))
    check(st, "dd_gemm")
    return out


def _shared_stride(ts, name):
    """The row stride of matrices of one shape, or None where they differ."""
    for t in ts:
        _mat(t, name)
        if t.shape != ts[0].shape:
            raise ValueError(f"the {name} matrices must agree in shape")
    strides = {t.stride(0) for t in ts}
    return strides.pop() if len(strides) == 1 else None


def _same(ts, name):
    """Matrices of one shape and row stride; returns that stride."""
    ld = _shared_stride(ts, name)
    if ld is None:
        raise ValueError(f"the {name} matrices must agree in row stride")
    return ld


def _array(ts):
    return (ctypes.c_void_p * len(ts))(*(t.data_ptr() for t in ts))


def gemm_group(a, bs, trans_a: bool = False, trans_b: bool = False, outs=None):
    """[op(a) @ op(b) for b in bs] in one launch (at most three of one shape)."""
    _mat(a, "a")
    ldb = _same(bs, "b")
    M, K = (a.shape[1], a.shape[0]) if trans_a else (a.shape[0], a.shape[1])
    Kb, N = (bs[0].shape[1], bs[0].shape[0]) if trans_b else (bs[0].shape[0], bs[0].shape[1])
    if K != Kb:
        raise ValueError(f"inner dimensions differ: {K} vs {Kb}")
    n = len(bs)
    if outs is None:
        outs = [torch.empty((M, N), dtype=torch.bfloat16, device=a.device) for _ in bs]
    ldc = _same(outs, "out")
    if len(outs) != n or tuple(outs[0].shape) != (M, N):
        raise ValueError(f"need {n} outputs of shape {(M, N)}")
    need = lib().dd_gemm_group_workspace_bytes(M, N, K, n)
    ws = torch.empty(need, dtype=torch.uint8, device=a.device) if need else None
    st = lib().dd_gemm_group(_p(a), a.stride(0), int(bool(trans_a)), _array(bs), ldb,
                             int(bool(trans_b)), _array(outs), ldc, n, M, N, K, _p(ws), need,
                             _stream(a.device))
    check(st, "dd_gemm_group")
    return outs


def gemm_sum(as_, bs, trans_b: bool = False):
    """sum of a @ op(b) over the pairs of as_ and bs (at most three), summed in
    fp32 and rounded once.  The launch takes one row stride per side: where they
    differ, the products run one by one, each rounded as it is added."""
    lda, ldb = _shared_stride(as_, "a"), _shared_stride(bs, "b")
    M, K = as_[0].shape
    Kb, N = (bs[0].shape[1], bs[0].shape[0]) if trans_b else (bs[0].shape[0], bs[0].shape[1])
    if K != Kb or len(as_) != len(bs) or len(as_) > 3:
        raise ValueError("need at most three pairs that agree in their inner dimension")
    if lda is None or ldb is None:
        out = gemm(as_[0], bs[0], trans_b=trans_b)
        for a, b in zip(as_[1:], bs[1:]):
            gemm(a, b, trans_b=trans_b, residual=out, out=out)
        return out
    out = torch.empty((M, N), dtype=torch.bfloat16, device=as_[0].device)
    st = lib().dd_gemm_sum(_array(as_), lda, _array(bs), ldb, int(bool(trans_b)), _p(out), N,
                           len(as_), M, N, K, _stream(out.device))
    check(st, "dd_gemm_sum")
    return out


def gemm_swiglu(x, w1, w3):
    """(u, v, silu(u) * v) with u = x @ w1 and v = x @ w3, in one launch
    (one each where the row strides of w1 and w3 differ)."""
    _mat(x, "x")
    ldw = _shared_stride([w1, w3], "w")
    (M, K), (Kw, N) = x.shape, w1.shape
    if K != Kw:
        raise ValueError(f"inner dimensions differ: {K} vs {Kw}")
    if ldw is None:
        u, v = gemm(x, w1), gemm(x, w3)
        return u, v, swiglu(u, v)
    u, v, y = (torch.empty((M, N), dtype=torch.bfloat16, device=x.device) for _ in range(3))
    st = lib().dd_gemm_swiglu(_p(x), x.stride(0), _p(w1), _p(w3), ldw, _p(u), _p(v), _p(y), N,
                              M, N, K, _stream(x.device))
    check(st, "dd_gemm_swiglu")
    return u, v, y


def gemm_swiglu_backward(dy, w, u, v):
    """(du, dv) of silu(u) * v for the upstream gradient dy @ w.T, in one launch."""
    _mat(dy, "dy")
    _mat(w, "w")
    ldu = _same([u, v], "u")
    (M, K), (N, Kw) = dy.shape, w.shape
    if K != Kw or tuple(u.shape) != (M, N):
        raise ValueError("the shapes of dy, w and u do not agree")
    if ldu != N:
        raise ValueError("u and v must be contiguous")
    du, dv = torch.empty_like(u), torch.empty_like(v)
    st = lib().dd_gemm_swiglu_bwd(_p(dy), dy.stride(0), _p(w), w.stride(0), _p(u), _p(v), _p(du),
                                  _p(dv), N, M, N, K, _stream(dy.device))
    check(st, "dd_gemm_swiglu_bwd")
    return du, dv


def transpose(x, out=None):
    """x.T as a bf16 matrix with unit column stride (into ``out`` if given)."""
    _mat(x, "x")
    R, C = x.shape
    if out is None:
        out = torch.empty((C, R), dtype=torch.bfloat16, device=x.device)
    _mat(out, "out")
    if tuple(out.shape) != (C, R):
        raise ValueError(f"out has shape {tuple(out.shape)}, expected {(C, R)}")
    st = lib().dd_transpose(_p(x), x.stride(0), _p(out), out.stride(0), R, C,
                            _stream(x.device))
    check(st, "dd_transpose")
    return out


def layer_norm(x, w, b, eps: float = LN_EPS):
    """(y, mean, rstd) of LayerNorm over the rows of x [rows, d]."""
    _mat(x, "x")
    rows, d = x.shape
    if not x.is_contiguous():
        raise ValueError("x must be contiguous")
    y = torch.empty_like(x)
    mean = torch.empty(rows, dtype=torch.float32, device=x.device)
    rstd = torch.empty(rows, dtype=torch.float32, device=x.device)
    st = lib().dd_layernorm_fwd(_p(x), _p(w), _p(b), _p(y), _p(mean), _p(rstd), rows, d,
                                float(eps), _stream(x.device))
    check(st, "dd_layernorm_fwd")
    return y, mean, rstd


def layer_norm_backward(x, w, mean, rstd, dy, dres=None):
    """(dx, dw, db) of LayerNorm; ``dres`` (optional) is added to dx."""
    rows, d = x.shape
    dx = torch.empty_like(x)
    dw = torch.empty(d, dtype=torch.bfloat16, device=x.device)
    db = torch.empty(d, dtype=torch.bfloat16, device=x.device)
    need = lib().dd_layernorm_bwd_workspace_bytes(rows, d)
    ws = torch.empty(max(need, 16), dtype=torch.uint8, device=x.device)
    st = lib().dd_layernorm_bwd(_p(x), _p(w), _p(mean), _p(rstd), _p(dy.contiguous()),
                                _p(dres), _p(dx), _p(dw), _p(db), rows, d, _p(ws), ws.numel(),
                                _stream(x.device))
    check(st, "dd_layernorm_bwd")
    return dx, dw, db


def swiglu(u, v):
    """silu(u) * v elementwise."""
    y = torch.empty_like(u)
    st = lib().dd_swiglu_fwd(_p(u), _p(v), _p(y), u.numel(), _stream(u.device))
    check(st, "dd_swiglu_fwd")
    return y


def swiglu_backward(u, v, dy):
    """(du, dv) of y = silu(u) * v."""
    du, dv = torch.empty_like(u), torch.empty_like(v)
    st = lib().dd_swiglu_bwd(_p(u), _p(v), _p(dy.contiguous()), _p(du), _p(dv), u.numel(),
                             _stream(u.device))
    check(st, "dd_swiglu_bwd")
    return du, dv


# ---------------------------------------------------------------------------
# rows in 8 bits


@functools.lru_cache(maxsize=None)
def _entry(name):
    return getattr(lib(), name)


def _call(dev, name, *args):
    """Runs an entry point on the current stream of ``dev``."""
    if dev.index == torch._C._cuda_getDevice():
        st = _entry(name)(*args, _stream(dev))
    else:
        with torch.cuda.device(dev):
            st = _entry(name)(*args, _stream(dev))
    if st:
        check(st, name)


def _need(dev, name, *sizes):
    """Workspace bytes of a call on ``dev`` (its CUs are counted)."""
    if dev.index == torch._C._cuda_getDevice():
        return _entry(name)(*sizes)
    with torch.cuda.device(dev):
        return _entry(name)(*sizes)


def _dims(t, name, dtype, dev=None):
    """(rows, columns, row stride) of a matrix of this type with unit column
    stride on ``dev`` (any GPU if None).  A single row's stride, which is
    never used, is its length.  (Called some times per call of a few
    microseconds: one look at everything, and the reasons only on failure.)"""
    if isinstance(t, torch.Tensor) and t.dtype is dtype and t.dim() == 2:
        (rows, cols), (ld, one) = t.shape, t.stride()
        where = t.device
        if (one == 1 and not (rows | cols) >> 31  # int in the C ABI
                and (where == dev if dev is not None else where.type == "cuda")):
            return rows, cols, ld if rows > 1 else cols
    if not isinstance(t, torch.Tensor) or t.dim() != 2:
        raise ValueError(f"{name} must be a 2-D tensor")
    if t.device.type != "cuda" or t.dtype is not dtype:
        kind = "bf16" if dtype is torch.bfloat16 else "int8"
        raise ValueError(f"{name} must be a {kind} GPU tensor")
    if t.stride(1) != 1:
        raise ValueError(f"{name} must have unit column stride")
    if max(t.shape) >> 31:
        raise ValueError(f"{name} has 2^31 rows or columns or more: {tuple(t.shape)}")
    raise ValueError(f"{name} is on {t.device}, not on {dev}")


def _vec(t, name, n, dtype, dev):
    if (isinstance(t, torch.Tensor) and t.dtype is dtype and t.shape == (n,)
            and t.device == dev and t.is_contiguous()):
        return
    raise ValueError(f"{name} must be a contiguous {dtype} tensor of {n} elements on {dev}")


def _rows(t, name, shape, dev):
    """Checks a contiguous bf16 matrix of this shape on ``dev``."""
    rows, cols, ld = _dims(t, name, torch.bfloat16, dev)
    if (rows, cols) != shape:
        raise ValueError(f"{name} has shape {(rows, cols)}, expected {shape}")
    if ld != cols:
        raise ValueError(f"{name} must be contiguous")


def _result(out, rows, cols, dev, name="out"):
    """(``out`` or a new bf16 matrix, its row stride)."""
    if out is None:
        return torch.empty((rows, cols), dtype=torch.bfloat16, device=dev), cols
    r, c, ld = _dims(out, name, torch.bfloat16, dev)
    if (r, c) != (rows, cols):
        raise ValueError(f"{name} has shape {(r, c)}, expected {(rows, cols)}")
    return out, ld


def _norm_inputs(x, w, residual):
    """(rows, columns, x's row stride, the residual's, x + residual to be)."""
    rows, d, ldx = _dims(x, "x", torch.bfloat16)
    if not d:
        raise ValueError("the rows of x are empty")
    _vec(w, "w", d, torch.bfloat16, x.device)
    if residual is None:
        return rows, d, ldx, 0, None
    r, c, ldr = _dims(residual, "residual", torch.bfloat16, x.device)
    if (r, c) != (rows, d):
        raise ValueError("residual must match x in shape")
    return rows, d, ldx, ldr, torch.empty_like(x)


def rms_norm(x, w, residual=None, eps: float = LN_EPS):
    """(y, h, rstd) of RMSNorm over the rows of h = x + residual (rounded to
    bf16; x itself without one): rstd = 1 / sqrt(mean(h^2) + eps), y = h rstd w."""
    rows, d, ldx, ldr, h = _norm_inputs(x, w, residual)
    dev = x.device
    y = torch.empty_like(x)
    rstd = torch.empty(rows, dtype=torch.float32, device=dev)
    if rows:
        _call(dev, "dd_rmsnorm_fwd", _p(x), ldx, _p(residual), ldr, _p(w), _p(h), _p(y),
              _p(rstd), rows, d, eps)
    return y, x if h is None else h, rstd


def rms_norm_int8(x, w, residual=None, eps: float = LN_EPS):
    """(codes, scales, h, rstd): ``rms_norm`` with its output as codes."""
    rows, d, ldx, ldr, h = _norm_inputs(x, w, residual)
    dev = x.device
    codes = torch.empty_like(x, dtype=torch.int8)
    scales = torch.empty(rows, dtype=torch.float32, device=dev)
    rstd = torch.empty_like(scales)
    if rows:
        _call(dev, "dd_rmsnorm_int8_fwd", _p(x), ldx, _p(residual), ldr, _p(w), _p(h), _p(codes),
              d, _p(scales), _p(rstd), rows, d, eps)
    return codes, scales, x if h is None else h, rstd


def rms_norm_backward(h, w, rstd, dy, dres=None):
    """(dx, dw) of either norm for the gradient dy of its output; dx is the
    gradient of x and of the residual, ``dres`` (optional, the gradient of h
    from its other uses) is added to it.  Contiguous matrices."""
    rows, d, _ = _dims(h, "h", torch.bfloat16)
    dev = h.device
    _rows(h, "h", (rows, d), dev)
    _vec(w, "w", d, torch.bfloat16, dev)
    _vec(rstd, "rstd", rows, torch.float32, dev)
    _rows(dy, "dy", (rows, d), dev)
    if dres is not None:
        _rows(dres, "dres", (rows, d), dev)
    dx, dw = torch.empty_like(h), torch.empty_like(w)
    if not (rows and d):
        return dx, dw.zero_()
    need = _need(dev, "dd_rmsnorm_bwd_workspace_bytes", rows, d)
    ws = torch.empty(need, dtype=torch.uint8, device=dev)
    _call(dev, "dd_rmsnorm_bwd", _p(h), _p(w), _p(rstd), _p(dy), _p(dres), _p(dx), _p(dw), rows,
          d, _p(ws), need)
    return dx, dw


def quantize(x):
    """(codes, scales) of the rows of a bf16 matrix."""
    rows, d, ldx = _dims(x, "x", torch.bfloat16)
    codes = torch.empty_like(x, dtype=torch.int8)
    scales = torch.empty(rows, dtype=torch.float32, device=x.device)
    if not d:
        return codes, scales.zero_()
    if rows:
        _call(x.device, "dd_quantize", _p(x), ldx, _p(codes), d, _p(scales), rows, d)
    return codes, scales


def dequantize(codes, scales, out=None):
    """The bf16 values of codes (into ``out`` if given)."""
    rows, d, ldq = _dims(codes, "codes", torch.int8)
    dev = codes.device
    _vec(scales, "scales", rows, torch.float32, dev)
    out, ldy = _result(out, rows, d, dev)
    if rows and d:
        _call(dev, "dd_dequantize", _p(codes), ldq, _p(scales), _p(out), ldy, rows, d)
    return out


def gemm_int8(a, a_scales, b, b_scales, residual=None, out=None):
    """(a_scales * a) @ (b_scales * b).T (+ residual) in bf16, from codes a
    [M, K] (tokens) and b [N, K] (output channels; a weight W [K, N] is kept
    as ``quantize(W.T.contiguous())``), K a multiple of 16 below 2^17.

    The sums are exact, scaled in fp32 and rounded once.  ``out`` (optional)
    receives the result and may be ``residual`` itself.  (``quantize`` forms
    codes of K up to 16384; longer rows are a caller's own.)"""
    M, K, lda = _dims(a, "a", torch.int8)
    dev = a.device
    N, Kb, ldb = _dims(b, "b", torch.int8, dev)
    if Kb != K:
        raise ValueError(f"inner dimensions differ: {K} vs {Kb}")
    if K % 16 or not 0 < K < 1 << 17:
        raise ValueError(f"the inner dimension must be a multiple of 16 below 2^17 (got {K})")
    _vec(a_scales, "a_scales", M, torch.float32, dev)
    _vec(b_scales, "b_scales", N, torch.float32, dev)
    out, ldc = _result(out, M, N, dev)
    if residual is not None and _dims(residual, "residual", torch.bfloat16, dev) != (M, N, ldc):
        raise ValueError("residual must match out in shape and row stride")
    if M and N:
        _call(dev, "dd_gemm_i8", _p(a), lda, _p(a_scales), _p(b), ldb, _p(b_scales), _p(residual),
              _p(out), ldc, M, N, K)
    return out


def gemm_int8_wgrad(codes, scales, dy, out=None):
    """``dequantize(codes, scales).T @ dy``: the weight gradient [M, N] of a
    linear layer from its input, kept as codes [T, M], and the gradient dy
    [T, N] of its output; M and N multiples of 8."""
    return gemm_int8_wgrad_group(codes, scales, [dy], None if out is None else [out])[0]


def gemm_int8_wgrad_group(codes, scales, dys, outs=None):
    """``gemm_int8_wgrad`` of layers that share their input: one result for
    each of dys (one to three of one shape and row stride), in one launch."""
    T, M, ldq = _dims(codes, "codes", torch.int8)
    dev, n = codes.device, len(dys)
    _vec(scales, "scales", T, torch.float32, dev)
    if not 1 <= n <= 3:
        raise ValueError(f"need one to three gradients (got {n})")
    shapes = [_dims(dy, "dy", torch.bfloat16, dev) for dy in dys]
    Ty, N, ldy = shapes[0]
    if any(s != shapes[0] for s in shapes):
        raise ValueError("the dy matrices must agree in shape and row stride")
    if Ty != T:
        raise ValueError(f"codes have {T} rows, dy has {Ty}")
    if M % 8 or N % 8:
        raise ValueError(f"the columns of codes and dy must be multiples of 8 (got {M} and {N})")
    if outs is None:
        outs = [None] * n
    elif len(outs) != n:
        raise ValueError(f"need {n} outputs of shape {(M, N)}")
    results = [_result(out, M, N, dev) for out in outs]
    outs, ldw = [out for out, _ in results], results[0][1]
    if any(ld != ldw for _, ld in results):
        raise ValueError("the outputs must agree in row stride")
    if not T:
        return [out.zero_() for out in outs]
    if M and N:
        need = _need(dev, "dd_gemm_i8_wgrad_workspace_bytes", T, M, N, n)
        ws = torch.empty(need, dtype=torch.uint8, device=dev)
        _call(dev, "dd_gemm_i8_wgrad", _p(codes), ldq, _p(scales), _array(dys), ldy, _array(outs),
              ldw, n, T, M, N, _p(ws), need)
    return outs

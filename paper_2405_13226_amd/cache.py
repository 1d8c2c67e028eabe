"""A paged cache of keys and values, and the attention that reads it: what a
model trained with this package generates with, or scores long texts in pieces.

Argument marshalling only, as in ``attention.py``; the kernels are behind the
dd_cache_* functions of include/dd_attn.h.

    k_pages, v_pages   bf16 [pages, kv heads, page, D], contiguous; page a power
                       of two in 16 .. 1024
    table              int32 [B, pages per sequence]: slot j of sequence b is
                       row j % page of page table[b, j // page]
    lens               int32 [B]: slots in use before the call
    cu_new             int32 [B + 1]: rows cu_new[b] .. cu_new[b + 1] of the
                       chunk are sequence b's new tokens, in slots lens[b] on
    weights            fp32 [B, kv heads, slots]: a slot's attention
                       probabilities, summed over the tokens so far and the
                       heads that share the key head
    positions          int32, of the same shape: a slot's position

Query rows are bf16 [T, H, D], H a multiple of the kv heads, a token's heads
contiguous (columns of a wider matrix are fine).  Rows behind cu_new[B] are left
as they were.  The calls read these tensors on the device and check their types
and shapes only: ``check_cache`` checks the contents of host copies.  Calls run
on the tensors' device, on its current stream, allocate only their results and
scratch, and can be captured in a graph.

``PagedCache`` keeps all of it for one layer.
"""
from __future__ import annotations

import ctypes

import numpy as np
import torch

from ._lib import check, lib
from .attention import _ptr as _p
from .block_ops import _call, _need


def _rows3(t, name, dev=None, heads=None, dim=None):
    """(T, heads, D, token stride) of a chunk's bf16 rows."""
    if isinstance(t, torch.Tensor) and t.dtype is torch.bfloat16 and t.dim() == 3:
        T, H, D = t.shape
        ld, sh, one = t.stride()
        if T <= 1:
            ld = H * D
        if ((one == 1 or D == 1) and (sh == D or H == 1) and ld >= H * D
                and (t.device == dev if dev is not None else t.is_cuda)
                and (heads is None or H == heads) and (dim is None or D == dim)):
            return T, H, D, ld
    if not isinstance(t, torch.Tensor) or t.dim() != 3:
        raise ValueError(f"{name} must be a 3-D tensor [tokens, heads, D]")
    if t.dtype is not torch.bfloat16 or not t.is_cuda:
        raise ValueError(f"{name} must be a bf16 GPU tensor")
    if dev is not None and t.device != dev:
        raise ValueError(f"{name} is on {t.device}, not on {dev}")
    if (heads is not None and t.shape[1] != heads) or (dim is not None and t.shape[2] != dim):
        raise ValueError(f"{name} has shape {tuple(t.shape)}, expected [tokens, {heads}, {dim}]")
    raise ValueError(f"the heads of a token of {name} must be contiguous (strides {t.stride()})")


def _pages(k_pages, v_pages, dev=None):
    """(pages, kv heads, page, D) of a cache."""
    for t, name in ((k_pages, "k_pages"), (v_pages, "v_pages")):
        if not (isinstance(t, torch.Tensor) and t.dim() == 4 and t.dtype is torch.bfloat16
                and t.is_cuda and t.is_contiguous()):
            raise ValueError(f"{name} must be a contiguous bf16 GPU tensor "
                             "[pages, kv heads, page, D]")
        if dev is not None and t.device != dev:
            raise ValueError(f"{name} is on {t.device}, not on {dev}")
    if k_pages.shape != v_pages.shape or k_pages.device != v_pages.device:
        raise ValueError("k_pages and v_pages must agree in shape and device")
    return k_pages.shape


def _state(t, name, shape, dtype, dev):
    if (isinstance(t, torch.Tensor) and t.dtype is dtype and t.shape == shape and t.device == dev
            and t.is_contiguous()):
        return
    raise ValueError(f"{name} must be a contiguous {dtype} tensor of shape {tuple(shape)} on {dev}")


def _table(table, lens, dev):
    """(B, pages per sequence)."""
    if not (isinstance(table, torch.Tensor) and table.dim() == 2):
        raise ValueError("table must be a 2-D tensor [B, pages per sequence]")
    B, per = table.shape
    _state(table, "table", (B, per), torch.int32, dev)
    _state(lens, "lens", (B,), torch.int32, dev)
    return B, per


def check_cache(table, lens, cu_new=None, pages=None, page=64, tokens=None) -> None:
    """Checks host copies of a cache's contents (lists, numpy arrays or
    tensors, which are copied): offsets in order and at most ``tokens`` of them,
    slots within the table, every page in use named once.  Raises DDError."""
    def host(x):
        x = x.detach().cpu().numpy() if isinstance(x, torch.Tensor) else np.asarray(x)
        if x.size and (x.max() >= 2 ** 31 or x.min() < -2 ** 31):
            raise ValueError("cache contents must fit int32")
        return np.ascontiguousarray(x, dtype=np.int32)

    table, lens = host(table), host(lens)
    if table.ndim != 2 or lens.shape != table.shape[:1]:
        raise ValueError("table must be [B, pages per sequence] and lens [B]")
    cu = None if cu_new is None else host(cu_new)
    if cu is not None and cu.shape != (len(lens) + 1,):
        raise ValueError("cu_new needs B + 1 offsets")
    if pages is None:
        pages = max(int(table.max(initial=0)) + 1, 1)
    if tokens is None:
        tokens = int(cu[-1]) if cu is not None else 0
    p = [x.ctypes.data_as(ctypes.c_void_p) if x is not None else None for x in (table, lens, cu)]
    check(lib().dd_cache_check(*p, tokens, *table.shape[:1], pages, page, table.shape[1]),
          "dd_cache_check")


def cache_append(q, k, v, k_pages, v_pages, table, lens, cu_new, rope_base=None, start=None,
                 positions=None, out=None):
    """Writes the chunk's k and v [T, kv heads, D] into their slots and returns
    q.  With ``rope_base`` q and k are rotated first (new tensor, or ``out``,
    which may be a contiguous q; q may be None), new token i of sequence b at
    position start[b] + i (int32 [B]; its slot without ``start``).
    ``positions`` (optional) receives the position of each written slot."""
    T, Hkv, D, ldk = _rows3(k, "k")
    dev = k.device
    ldv = _rows3(v, "v", dev, Hkv, D)[3]
    if v.shape[0] != T:
        raise ValueError(f"k has {T} tokens, v has {v.shape[0]}")
    pages, heads, page, dim = _pages(k_pages, v_pages, dev)
    if (heads, dim) != (Hkv, D):
        raise ValueError(f"k has {Hkv} heads of {D}, the pages {heads} of {dim}")
    B, per = _table(table, lens, dev)
    _state(cu_new, "cu_new", (B + 1,), torch.int32, dev)
    if start is not None:
        _state(start, "start", (B,), torch.int32, dev)
    if positions is not None:
        _state(positions, "positions", (B, Hkv, per * page), torch.int32, dev)
    H, ldq, rot = Hkv, 0, None
    if q is not None:
        Tq, H, _, ldq = _rows3(q, "q", dev, None, D)
        if Tq != T:
            raise ValueError(f"q has {Tq} tokens, k has {T}")
    if rope_base is not None and q is not None:
        if out is None:
            out = torch.empty((T, H, D), dtype=torch.bfloat16, device=dev)
        else:
            _state(out, "out", (T, H, D), torch.bfloat16, dev)
        rot = out
    elif out is not None:
        raise ValueError("out is the rotated q: it needs rope_base and q")
    if rope_base is not None and not rope_base > 0:
        raise ValueError(f"rope_base must be positive (got {rope_base})")
    if T and B:
        _call(dev, "dd_cache_append", _p(q) if rot is not None else None, ldq, _p(k), ldk, _p(v),
              ldv, _p(rot), _p(k_pages), _p(v_pages), _p(positions), _p(table), _p(lens), _p(start),
              _p(cu_new), T, B, H, Hkv, D, pages, page, per, rope_base or 0.0)
    return q if rot is None else rot


def cache_attention(q, k_pages, v_pages, table, lens, cu_new, weights=None, weights_out=None,
                    out=None, lse=None):
    """(o [T, H, D] bf16, lse [T, H] fp32) of the chunk's queries over the
    cache, to which its keys and values were appended: new token i of sequence
    b sees slots 0 .. lens[b] + i.  ``weights`` (optional) is brought up to date
    in place, or into ``weights_out``.  ``out`` and ``lse`` receive the results
    if given (both, or neither)."""
    T, H, D, ldq = _rows3(q, "q")
    dev = q.device
    pages, Hkv, page, dim = _pages(k_pages, v_pages, dev)
    if dim != D or not Hkv or H % Hkv:
        raise ValueError(f"q has {H} heads of {D}, the pages {Hkv} of {dim}")
    B, per = _table(table, lens, dev)
    _state(cu_new, "cu_new", (B + 1,), torch.int32, dev)
    if weights is not None:
        _state(weights, "weights", (B, Hkv, per * page), torch.float32, dev)
    if weights_out is not None:
        if weights is None:
            raise ValueError("weights_out needs weights")
        _state(weights_out, "weights_out", (B, Hkv, per * page), torch.float32, dev)
    if (out is None) != (lse is None):
        raise ValueError("give both out and lse, or neither")
    if out is None:
        out = torch.empty((T, H, D), dtype=torch.bfloat16, device=dev)
        lse = torch.empty((T, H), dtype=torch.float32, device=dev)
    else:
        _state(out, "out", (T, H, D), torch.bfloat16, dev)
        _state(lse, "lse", (T, H), torch.float32, dev)
    if not (T and B):
        if weights_out is not None and weights_out is not weights:
            weights_out.copy_(weights)
        return out, lse
    need = _need(dev, "dd_cache_attn_workspace_bytes", T, B, H, Hkv, D, page, per,
                 weights is not None)
    ws = torch.empty(need, dtype=torch.uint8, device=dev) if need else None
    _call(dev, "dd_cache_attn_fwd", _p(q), ldq, _p(k_pages), _p(v_pages), _p(table), _p(lens),
          _p(cu_new), _p(out), _p(lse), _p(weights),
          _p(weights if weights_out is None else weights_out), T, B, H, Hkv, D, pages, page, per,
          _p(ws), need)
    return out, lse


def cache_evict(k_pages, v_pages, table, lens, weights, positions, seen, budget: int,
                recent: int = 0, out=None):
    """Thins each sequence and key head out to the ``budget`` slots of most
    weight: slots whose position is at least seen[b] - recent (seen: int32 [B],
    the position after the last) stay before all others, a NaN counts least,
    equal weights go by the lowest slot.  Keys and values move within the pages:
    the n-th slot below the budget that goes receives the n-th one behind it
    that stays.  Returns (weights, positions, lens) of the slots that are left
    (new tensors, defined up to the new lens, or ``out``: three tensors, each of
    which may be the input itself)."""
    pages, Hkv, page, D = _pages(k_pages, v_pages)
    dev = k_pages.device
    B, per = _table(table, lens, dev)
    _state(weights, "weights", (B, Hkv, per * page), torch.float32, dev)
    _state(positions, "positions", (B, Hkv, per * page), torch.int32, dev)
    _state(seen, "seen", (B,), torch.int32, dev)
    if not 0 <= recent <= budget or budget < 1:
        raise ValueError(f"need 0 <= recent <= budget and a budget of at least 1 "
                         f"(got {recent} and {budget})")
    budget = min(int(budget), max(per * page, 1))
    if out is None:
        out = tuple(torch.empty_like(t) for t in (weights, positions, lens))
    else:
        out = tuple(out)
        for t, like, name in zip(out, (weights, positions, lens), ("weights", "positions", "lens")):
            _state(t, "out " + name, like.shape, like.dtype, dev)
        if len(out) != 3:
            raise ValueError("out must hold weights, positions and lens")
    if B and Hkv and per:
        need = _need(dev, "dd_cache_evict_workspace_bytes", B, Hkv, D, page, per, budget)
        ws = torch.empty(max(need, 4), dtype=torch.uint8, device=dev)
        _call(dev, "dd_cache_evict", _p(k_pages), _p(v_pages), _p(table), _p(lens), _p(weights),
              _p(positions), _p(seen), *(_p(t) for t in out), B, Hkv, D, pages, page, per, budget,
              min(int(recent), budget), _p(ws), need)
    return out


class PagedCache:
    """Keys and values of one layer for a batch of sequences: the pages, each
    sequence's table, lengths and positions, and (``weights=True``) the slots'
    attention weights, which eviction needs.

    Lengths and pages in use are kept on the host as well, so that nothing has
    to be read back; a call that finds no free page raises RuntimeError and
    changes nothing."""

    def __init__(self, batch: int, kv_heads: int, dim: int, capacity: int, page: int = 64,
                 pages: int = None, weights: bool = False, device="cuda"):
        self.page, self.per = page, -(-capacity // page)
        pages = batch * self.per if pages is None else pages
        self.k_pages, self.v_pages = (
            torch.zeros((pages, kv_heads, page, dim), dtype=torch.bfloat16, device=device)
            for _ in range(2))
        self.lengths = [0] * batch  # slots in use
        self.tokens = [0] * batch   # tokens seen
        self.free = list(range(pages - 1, -1, -1))
        self.owned = [[] for _ in range(batch)]
        ints = dict(dtype=torch.int32, device=device)
        self.table = torch.full((batch, self.per), -1, **ints)
        self.lens, self.seen = torch.zeros(batch, **ints), torch.zeros(batch, **ints)
        shape = (batch, kv_heads, self.per * page)
        self.positions = torch.zeros(shape, **ints) if weights else None
        self.weights = torch.zeros(shape, dtype=torch.float32, device=device) if weights else None

    def _device_ints(self, values):
        return torch.tensor(values, dtype=torch.int32).to(self.table.device)

    def _set_tables(self):
        rows = [own + [-1] * (self.per - len(own)) for own in self.owned]
        self.table.copy_(self._device_ints(rows))

    def _reserve(self, news):
        slots = [n + m for n, m in zip(self.lengths, news)]
        if max(slots) > self.per * self.page:
            raise RuntimeError(f"a sequence would need {max(slots)} slots of "
                               f"{self.per * self.page}")
        more = [-(-n // self.page) - len(own) for n, own in zip(slots, self.owned)]
        need = sum(max(m, 0) for m in more)
        if need > len(self.free):
            raise RuntimeError(f"{need} pages needed, {len(self.free)} free")
        for own, m in zip(self.owned, more):
            own.extend(self.free.pop() for _ in range(max(m, 0)))
        if need:
            self._set_tables()

    def extend(self, q, k, v, news, rope_base=None, out=None, lse=None):
        """Appends the chunk (news[b] rows of sequence b, one after the other)
        and returns its attention (o, lse) over the cache."""
        news = [int(n) for n in news]
        if len(news) != len(self.lengths) or min(news, default=0) < 0:
            raise ValueError(f"need {len(self.lengths)} numbers of new tokens")
        if sum(news) > q.shape[0]:
            raise ValueError(f"{sum(news)} new tokens, but q has {q.shape[0]} rows")
        self._reserve(news)
        cu = self._device_ints(np.concatenate([[0], np.cumsum(news)]))
        q = cache_append(q, k, v, self.k_pages, self.v_pages, self.table, self.lens, cu,
                         rope_base=rope_base, start=self.seen, positions=self.positions)
        o, lse = cache_attention(q, self.k_pages, self.v_pages, self.table, self.lens, cu,
                                 weights=self.weights, out=out, lse=lse)
        self.lengths = [n + m for n, m in zip(self.lengths, news)]
        self.tokens = [n + m for n, m in zip(self.tokens, news)]
        step = cu[1:] - cu[:-1]
        self.lens += step
        self.seen += step
        return o, lse

    def evict(self, budget: int, recent: int = 0):
        """Thins every sequence out to ``budget`` slots and frees their pages."""
        if self.weights is None:
            raise ValueError("eviction needs a cache with weights=True")
        cache_evict(self.k_pages, self.v_pages, self.table, self.lens, self.weights, self.positions,
                    self.seen, budget, recent, out=(self.weights, self.positions, self.lens))
        self.lengths = [min(n, budget) for n in self.lengths]
        self._shrink()

    def clear(self, b: int):
        """Sequence b begins anew."""
        self.lengths[b] = self.tokens[b] = 0
        self.lens[b] = 0
        self.seen[b] = 0
        self._shrink()

    def _shrink(self):
        freed = False
        for n, own in zip(self.lengths, self.owned):
            while len(own) > -(-n // self.page):
                self.free.append(own.pop())
                freed = True
        if freed:
            self._set_tables()

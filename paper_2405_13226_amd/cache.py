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
and shapes only: ``check_cache`` checks the contents of host copies (it wants
every page in one sequence; attention, which only reads them, may be given
pages that sequences share).  Forward only.  Calls run
on the tensors' device, on its current stream, allocate only their results and
scratch, and can be captured in a graph.

``PagedCache`` keeps all of it for one layer.
"""
from __future__ import annotations

import ctypes
import functools
import itertools

import numpy as np
import torch

from ._lib import check, lib
from .attention import _ptr as _p
from .block_ops import _call, _entry

_BF16, _F32, _I32 = torch.bfloat16, torch.float32, torch.int32


@functools.lru_cache(maxsize=1024)
def _bytes(name, *sizes):
    """Workspace bytes of a call: of its sizes alone (the latest 1024 of them: a
    program that scores texts has ever new numbers of rows)."""
    return _entry(name)(*sizes)


# A call for a few tokens takes a dozen microseconds, most of them here: each
# wrapper looks at all its tensors in one expression first, and asks the
# functions below only for the reason of a refusal.


def _is(t, shape, dtype, i):
    """Whether t is a contiguous tensor of this shape and type on device i."""
    return (t.dtype is dtype and t.shape == shape and t.get_device() == i and t.is_contiguous())


def _held(k, v, shape, i):
    """Whether k and v are the pages of a cache on device i."""
    return (k.dtype is _BF16 and v.dtype is _BF16 and k.shape == shape == v.shape
            and k.get_device() == i == v.get_device() and k.is_contiguous() and v.is_contiguous())


def _like(q, ld):
    """A new contiguous tensor of q's shape (the shorter call where q is one)."""
    return torch.empty_like(q) if ld == q.shape[1] * q.shape[2] else q.new_empty(q.shape)


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
    try:
        (T, Hkv, D), (ldk, hk, one_k), (ldv, hv, one_v) = k.shape, k.stride(), v.stride()
        pages, _, page, _ = k_pages.shape
        B, per = table.shape
        i = k.get_device()
        if T == 1:
            ldk = ldv = Hkv * D
        fine = (k.dtype is _BF16 and v.dtype is _BF16 and v.shape == k.shape and i >= 0
                and one_k == one_v == 1 and hk == hv == D and ldk >= Hkv * D <= ldv
                and v.get_device() == i and _held(k_pages, v_pages, (pages, Hkv, page, D), i)
                and table.dtype is _I32 and table.get_device() == i and table.is_contiguous()
                and _is(lens, (B,), _I32, i) and _is(cu_new, (B + 1,), _I32, i)
                and (start is None or _is(start, (B,), _I32, i))
                and (positions is None or _is(positions, (B, Hkv, per * page), _I32, i)))
    except (AttributeError, TypeError, ValueError):
        fine = False
    if not fine:
        T, Hkv, D, ldk = _rows3(k, "k")
        ldv = _rows3(v, "v", k.device, Hkv, D)[3]
        if v.shape[0] != T:
            raise ValueError(f"k has {T} tokens, v has {v.shape[0]}")
        pages, heads, page, dim = _pages(k_pages, v_pages, k.device)
        if (heads, dim) != (Hkv, D):
            raise ValueError(f"k has {Hkv} heads of {D}, the pages {heads} of {dim}")
        B, per = _table(table, lens, k.device)
        _state(cu_new, "cu_new", (B + 1,), _I32, k.device)
        if start is not None:
            _state(start, "start", (B,), _I32, k.device)
        if positions is not None:
            _state(positions, "positions", (B, Hkv, per * page), _I32, k.device)
    H, ldq, rot = Hkv, 0, None
    if q is not None:
        Tq, H, _, ldq = _rows3(q, "q", k.device, None, D)
        if Tq != T:
            raise ValueError(f"q has {Tq} tokens, k has {T}")
    if rope_base is None or q is None:
        if out is not None:
            raise ValueError("out is the rotated q: it needs rope_base and q")
        H = Hkv  # (q is not read)
    else:
        rot = _like(q, ldq) if out is None else out
        if out is not None:
            _state(out, "out", (T, H, D), _BF16, k.device)
    if rope_base is not None and not 2.0 ** -126 <= rope_base < 2.0 ** 128:
        raise ValueError(f"rope_base must be positive and fit fp32 (got {rope_base})")
    if T and B:
        _call(k.device, "dd_cache_append", q.data_ptr() if rot is not None else None, ldq,
              k.data_ptr(), ldk, v.data_ptr(), ldv, _p(rot), k_pages.data_ptr(),
              v_pages.data_ptr(), _p(positions), table.data_ptr(), lens.data_ptr(), _p(start),
              cu_new.data_ptr(), T, B, H, Hkv, D, pages, page, per, rope_base or 0.0)
    return q if rot is None else rot


def cache_attention(q, k_pages, v_pages, table, lens, cu_new, weights=None, weights_out=None,
                    out=None, lse=None):
    """(o [T, H, D] bf16, lse [T, H] fp32) of the chunk's queries over the
    cache, to which its keys and values were appended: new token i of sequence
    b sees slots 0 .. lens[b] + i.  ``weights`` (optional) is brought up to date
    in place, or into ``weights_out``.  ``out`` and ``lse`` receive the results
    if given (both, or neither)."""
    try:
        (T, H, D), (ldq, head, one) = q.shape, q.stride()
        pages, Hkv, page, _ = k_pages.shape
        B, per = table.shape
        i = q.get_device()
        if T == 1:
            ldq = H * D
        fine = (q.dtype is _BF16 and i >= 0 and one == 1 and head == D and ldq >= H * D and not H % Hkv
                and _held(k_pages, v_pages, (pages, Hkv, page, D), i)
                and table.dtype is _I32 and table.get_device() == i and table.is_contiguous()
                and _is(lens, (B,), _I32, i) and _is(cu_new, (B + 1,), _I32, i))
        if fine and weights is not None:
            slots = (B, Hkv, per * page)
            fine = _is(weights, slots, _F32, i) and (weights_out is None
                                                     or _is(weights_out, slots, _F32, i))
    except (AttributeError, TypeError, ValueError, ZeroDivisionError):
        fine = False
    if not fine:
        T, H, D, ldq = _rows3(q, "q")
        pages, Hkv, page, dim = _pages(k_pages, v_pages, q.device)
        if dim != D or not Hkv or H % Hkv:
            raise ValueError(f"q has {H} heads of {D}, the pages {Hkv} of {dim}")
        B, per = _table(table, lens, q.device)
        _state(cu_new, "cu_new", (B + 1,), _I32, q.device)
        for t, name in ((weights, "weights"), (weights_out, "weights_out")):
            if t is not None:
                _state(t, name, (B, Hkv, per * page), _F32, q.device)
    if weights_out is None:
        weights_out = weights
    elif weights is None:
        raise ValueError("weights_out needs weights")
    if (out is None) != (lse is None):
        raise ValueError("give both out and lse, or neither")
    dev = q.device
    if out is None:
        out = _like(q, ldq)
        lse = q.new_empty((T, H), dtype=_F32)
    else:
        _state(out, "out", (T, H, D), _BF16, dev)
        _state(lse, "lse", (T, H), _F32, dev)
    if not (T and B):
        if weights_out is not weights and B and per:  # the slots in use
            used = torch.arange(per * page, device=dev) < lens[:, None, None]
            weights_out.copy_(torch.where(used, weights, weights_out))
        return out, lse
    need = _bytes("dd_cache_attn_workspace_bytes", T, B, H, Hkv, D, page, per, weights is not None)
    ws = torch.empty(need, dtype=torch.uint8, device=dev) if need else None
    _call(dev, "dd_cache_attn_fwd", q.data_ptr(), ldq, k_pages.data_ptr(), v_pages.data_ptr(),
          table.data_ptr(), lens.data_ptr(), cu_new.data_ptr(), out.data_ptr(), lse.data_ptr(),
          _p(weights), _p(weights_out), T, B, H, Hkv, D, pages, page, per, _p(ws), need)
    return out, lse


def cache_evict(k_pages, v_pages, table, lens, weights, positions, seen, budget: int,
                recent: int = 0, out=None):
    """Thins each sequence and key head out to the ``budget`` slots of most
    weight: slots whose position is at least seen[b] - recent (seen: int32 [B],
    the position after the last) stay before all others, a NaN counts least,
    equal weights go by the lowest slot.  Keys and values move within the pages:
    the n-th slot below the budget that goes receives the n-th one behind it
    that stays.  Returns (weights, positions, lens) of the slots that are left
    (new tensors, or ``out``: three tensors, each of which may be the input
    itself); weights and positions hold the first ``budget`` slots, behind the
    new lens what the inputs hold there, and are not written behind the budget."""
    try:
        pages, Hkv, page, D = shape = k_pages.shape
        B, per = table.shape
        i = k_pages.get_device()
        slots = (B, Hkv, per * page)
        fine = (i >= 0 and _held(k_pages, v_pages, shape, i)
                and table.dtype is _I32 and table.get_device() == i and table.is_contiguous()
                and _is(lens, (B,), _I32, i) and _is(seen, (B,), _I32, i)
                and _is(weights, slots, _F32, i) and _is(positions, slots, _I32, i))
    except (AttributeError, TypeError, ValueError):
        fine = False
    if not fine:
        pages, Hkv, page, D = _pages(k_pages, v_pages)
        dev = k_pages.device
        B, per = _table(table, lens, dev)
        _state(weights, "weights", (B, Hkv, per * page), _F32, dev)
        _state(positions, "positions", (B, Hkv, per * page), _I32, dev)
        _state(seen, "seen", (B,), _I32, dev)
    if not 0 <= recent <= budget or budget < 1:
        raise ValueError(f"need 0 <= recent <= budget and a budget of at least 1 "
                         f"(got {recent} and {budget})")
    budget = min(int(budget), max(per * page, 1))
    recent = min(int(recent), budget)
    dev = k_pages.device
    if out is None:
        w, p, n = torch.empty_like(weights), torch.empty_like(positions), torch.empty_like(lens)
    else:
        w, p, n = out
        for t, like, name in ((w, weights, "weights"), (p, positions, "positions"),
                              (n, lens, "lens")):
            _state(t, "out " + name, like.shape, like.dtype, dev)
    if B and Hkv and per:
        in_place = n.data_ptr() == lens.data_ptr()
        need = _bytes("dd_cache_evict_workspace_bytes", B, Hkv, D, page, per, budget, in_place)
        ws = torch.empty(need, dtype=torch.uint8, device=dev) if need else None
        _call(dev, "dd_cache_evict", k_pages.data_ptr(), v_pages.data_ptr(), table.data_ptr(),
              lens.data_ptr(), weights.data_ptr(), positions.data_ptr(), seen.data_ptr(),
              w.data_ptr(), p.data_ptr(), n.data_ptr(), B, Hkv, D, pages, page, per, budget, recent,
              _p(ws), need)
    elif B:  # no heads, or no slots
        torch.clamp(lens, 0, budget if per else 0, out=n)
    return w, p, n


class PagedCache:
    """Keys and values of one layer for a batch of sequences: the pages, each
    sequence's table, lengths and positions, and (``weights=True``) the slots'
    attention weights, which eviction needs.

    Lengths and pages in use are kept on the host as well, so that nothing has
    to be read back; a call that finds no free page raises RuntimeError and
    changes nothing.  ``extend``, ``evict`` and ``clear`` bring the device's
    offsets and tables up to date from the host, which waits for the stream:
    they are not for a captured graph."""

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
        self.table.copy_(self._device_ints(rows).view(self.table.shape))

    def _reserve(self, news):
        slots = [n + m for n, m in zip(self.lengths, news)]
        if max(slots, default=0) > self.per * self.page:
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

    def counts(self, news):
        """The numbers of new tokens as a list, one for each sequence."""
        news = [int(n) for n in news]
        if len(news) != len(self.lengths) or min(news, default=0) < 0:
            raise ValueError(f"need {len(self.lengths)} numbers of new tokens")
        return news

    def extend(self, q, k, v, news, rope_base=None, out=None, lse=None):
        """Appends the chunk (news[b] rows of sequence b, one after the other)
        and returns its attention (o, lse) over the cache.  Rows behind the
        chunk's last are left as they were in ``out`` and ``lse``."""
        news = self.counts(news)
        rows, n = q.shape[0], sum(news)
        if n > rows:
            raise ValueError(f"{n} new tokens, but q has {rows} rows")
        if n < rows:
            return self._extend_first(q, k, v, news, rope_base, out, lse)
        self._reserve(news)
        cu = self._device_ints([0, *itertools.accumulate(news)])
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

    def _extend_first(self, q, k, v, news, rope_base, out, lse):
        """``extend`` where rows lie behind the chunk's: the operators, which
        choose their kernels by the number of rows, get the chunk's alone."""
        n, rows = sum(news), q.shape[0]
        for t, name in ((k, "k"), (v, "v")):
            if not isinstance(t, torch.Tensor) or t.shape[:1] != q.shape[:1]:
                raise ValueError(f"q has {rows} rows, {name} must have as many")
        if (out is None) != (lse is None):
            raise ValueError("give both out and lse, or neither")
        if out is None:
            out, lse = q.new_empty(q.shape), q.new_empty(q.shape[:2], dtype=_F32)
        else:
            _state(out, "out", q.shape, _BF16, q.device)
            _state(lse, "lse", q.shape[:2], _F32, q.device)
        self.extend(q[:n], k[:n], v[:n], news, rope_base, out[:n], lse[:n])
        return out, lse

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

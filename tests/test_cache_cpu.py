"""The paged cache and the log probabilities without a GPU: every refusal of the
C ABI (validation runs on the host before any launch), the checks of host
copies, and the Python wrappers' refusals."""
import ctypes

import numpy as np
import pytest
import torch

from paper_2405_13226_amd import _lib, cache, loss as lp

OK, NULL, SHAPE, HEADDIM, DOCLENS, WORKSPACE, ALIGN, ALIAS = range(8)
CACHE = 10
GiB = 1 << 30


def fake(i, off=0):
    """Addresses 2^36 apart; never read."""
    return ctypes.c_void_p((i + 1) * (1 << 36) + off)


@pytest.fixture(scope="module")
def lib():
    return _lib.lib()


def call(lib, fn, defaults, **kw):
    a = dict(defaults)
    assert set(kw) <= set(a), kw
    a.update(kw)
    return getattr(lib, fn)(*a.values(), None)


SIZES = dict(T=8, B=2, H=4, Hkv=2, D=64, pages=10, page=16, per=5)
APPEND = dict(Q=fake(0), ldq=256, K=fake(1), ldk=128, V=fake(2), ldv=128, Qrot=fake(3), Kp=fake(4),
              Vp=fake(5), positions=fake(6), table=fake(7), lens=fake(8), start=fake(9),
              cu_new=fake(10), **SIZES, rope_base=1e4)
ATTN = dict(Q=fake(0), ldq=256, Kp=fake(4), Vp=fake(5), table=fake(7), lens=fake(8),
            cu_new=fake(10), O=fake(11), LSE=fake(12), W_in=fake(13), W_out=fake(14), **SIZES,
            ws=fake(15), bytes=1 << 30)
EVICT = dict(Kp=fake(4), Vp=fake(5), table=fake(7), lens=fake(8), W_in=fake(13), P_in=fake(6),
             seen=fake(9), W_out=fake(14), P_out=fake(16), lens_out=fake(17), B=2, Hkv=2, D=64,
             pages=10, page=16, per=5, budget=40, recent=8, ws=fake(15), bytes=1 << 30)


@pytest.mark.parametrize("fn,base", [("dd_cache_append", APPEND), ("dd_cache_attn_fwd", ATTN)])
def test_sizes_refused(lib, fn, base):
    for kw in (dict(T=0), dict(B=0), dict(H=0), dict(Hkv=0), dict(H=3), dict(pages=0), dict(per=0),
               dict(page=8), dict(page=24), dict(page=2048), dict(page=0), dict(per=1 << 27),
               dict(T=(1 << 23) + 1), dict(T=1 << 22, H=32, ldq=1 << 15),
               dict(B=40000), dict(ldq=248), dict(ldq=1 << 31), dict(T=-1), dict(B=-1)):
        assert call(lib, fn, base, **kw) == SHAPE, kw
    for D in (0, 32, 80, 256):
        assert call(lib, fn, base, D=D) == HEADDIM
    assert call(lib, fn, base, ldq=260) == ALIGN


def test_append_refusals(lib):
    for n in ("Q", "K", "V", "Qrot", "Kp", "Vp", "table", "lens", "cu_new"):
        assert call(lib, "dd_cache_append", APPEND, **{n: None}) == NULL, n
    for kw in (dict(ldk=120), dict(ldv=64), dict(rope_base=-1.0), dict(rope_base=float("inf")),
               dict(rope_base=float("nan")), dict(rope_base=0.0)):
        assert call(lib, "dd_cache_append", APPEND, **kw) == SHAPE, kw
    for n, off in (("Q", 8), ("K", 2), ("V", 4), ("Qrot", 8), ("Kp", 8), ("Vp", 2), ("positions", 2),
                   ("table", 1), ("lens", 2), ("start", 2), ("cu_new", 3)):
        i = APPEND[n].value // (1 << 36) - 1
        assert call(lib, "dd_cache_append", APPEND, **{n: fake(i, off)}) == ALIGN, n
    assert call(lib, "dd_cache_append", APPEND, ldk=132) == ALIGN
    for kw in (dict(Kp=fake(5)), dict(Kp=fake(1, 256)), dict(Vp=fake(0)), dict(Qrot=fake(0, 16)),
               dict(positions=fake(4)), dict(positions=fake(8)), dict(Qrot=fake(0), ldq=264)):
        assert call(lib, "dd_cache_append", APPEND, **kw) == ALIAS, kw


def test_attention_refusals(lib):
    for n in ("Q", "Kp", "Vp", "table", "lens", "cu_new", "O", "LSE", "W_in", "W_out"):
        assert call(lib, "dd_cache_attn_fwd", ATTN, **{n: None}) == NULL, n
    for n, off in (("Q", 8), ("Kp", 8), ("Vp", 2), ("O", 8), ("LSE", 2), ("W_in", 2), ("W_out", 1),
                   ("table", 1), ("lens", 2), ("cu_new", 3)):
        i = ATTN[n].value // (1 << 36) - 1
        assert call(lib, "dd_cache_attn_fwd", ATTN, **{n: fake(i, off)}) == ALIGN, n
    for kw in (dict(O=fake(0)), dict(O=fake(4)), dict(LSE=fake(11)), dict(W_out=fake(13, 4)),
               dict(W_out=fake(8)), dict(W_in=fake(12))):
        assert call(lib, "dd_cache_attn_fwd", ATTN, **kw) == ALIAS, kw
    big = dict(ATTN, per=640, pages=1280)
    need = lib.dd_cache_attn_workspace_bytes(8, 2, 4, 2, 64, 16, 640, 1)
    assert need >= lib.dd_cache_attn_workspace_bytes(8, 2, 4, 2, 64, 16, 640, 0) > 0
    assert call(lib, "dd_cache_attn_fwd", big, ws=None) == WORKSPACE
    assert call(lib, "dd_cache_attn_fwd", big, bytes=need - 1) == WORKSPACE
    assert call(lib, "dd_cache_attn_fwd", big, ws=fake(15, 8)) == ALIGN
    assert call(lib, "dd_cache_attn_fwd", big, ws=fake(11)) == ALIAS
    assert lib.dd_cache_attn_workspace_bytes(0, 2, 4, 2, 64, 16, 64, 0) == 0
    assert lib.dd_cache_attn_workspace_bytes(8, 2, 4, 2, 80, 16, 64, 1) == 0
    assert lib.dd_cache_attn_workspace_bytes(8, 2, 5, 2, 64, 16, 64, 0) == 0


def test_evict_refusals(lib):
    for n in ("Kp", "Vp", "table", "lens", "W_in", "P_in", "seen", "W_out", "P_out", "lens_out"):
        assert call(lib, "dd_cache_evict", EVICT, **{n: None}) == NULL, n
    for kw in (dict(B=0), dict(Hkv=0), dict(pages=0), dict(page=12), dict(per=0), dict(budget=0),
               dict(recent=-1), dict(recent=41), dict(B=40000), dict(budget=-3)):
        assert call(lib, "dd_cache_evict", EVICT, **kw) == SHAPE, kw
    assert call(lib, "dd_cache_evict", EVICT, D=96) == HEADDIM
    # lists for the moves: in place, or long
    assert lib.dd_cache_evict_workspace_bytes(2, 2, 64, 16, 5, 0, 1) == 0
    assert lib.dd_cache_evict_workspace_bytes(2, 2, 64, 16, 5, 40, 0) == 0
    for kw in (dict(lens_out=EVICT["lens"]), dict(per=200, pages=400, budget=1600)):
        args = {**EVICT, **kw}
        need = lib.dd_cache_evict_workspace_bytes(2, 2, 64, 16, args["per"], args["budget"],
                                                  int("lens_out" in kw))
        assert need > 0
        assert call(lib, "dd_cache_evict", args, ws=None) == WORKSPACE
        assert call(lib, "dd_cache_evict", args, bytes=need - 1) == WORKSPACE
        assert call(lib, "dd_cache_evict", args, ws=fake(15, 2)) == ALIGN
        assert call(lib, "dd_cache_evict", args, ws=fake(4)) == ALIAS
    for kw in (dict(W_out=fake(13, 4)), dict(P_out=fake(6, 8)), dict(lens_out=fake(8, 4)),
               dict(Kp=fake(5)), dict(W_out=fake(9)), dict(W_out=fake(6)),
               dict(P_out=fake(14))):
        assert call(lib, "dd_cache_evict", EVICT, **kw) == ALIAS, kw


def test_check_cache():
    table = [[3, 1, -1], [0, 7, 99]]
    cache.check_cache(table, [20, 5], [0, 3, 14], pages=8, page=16, tokens=14)
    cache.check_cache(table, [32, 0], pages=8, page=16)
    cache.check_cache(torch.tensor(table), np.array([20, 5]), torch.tensor([0, 3, 14]), 8, 16)
    for kw in (dict(lens=[-1, 5]), dict(lens=[33, 5], cu=[0, 0, 0]), dict(lens=[20, 33], cu=[0, 0, 0]),
               dict(lens=[20, 49], cu=[0, 0, 0]), dict(cu=[1, 3, 14]), dict(cu=[0, 5, 3]),
               dict(cu=[0, 3, 15]), dict(table=[[3, 3, 0], [0, 7, 9]]),
               dict(table=[[3, 1, 0], [1, 7, 9]]), dict(table=[[3, 8, 0], [0, 7, 9]]),
               dict(table=[[3, -1, 0], [0, 7, 9]])):
        with pytest.raises(_lib.DDError) as e:
            cache.check_cache(kw.get("table", table), kw.get("lens", [20, 5]),
                              kw.get("cu", [0, 3, 14]), pages=8, page=16, tokens=14)
        assert e.value.status == CACHE, kw
    with pytest.raises(_lib.DDError) as e:
        cache.check_cache(table, [20, 5], pages=8, page=24)
    assert e.value.status == SHAPE
    for args in (([1, 2], [3, 4]), (table, [1]), (table, [1, 2], [0, 1]), (table, [2 ** 31, 1])):
        with pytest.raises(ValueError):
            cache.check_cache(*args, pages=8, page=16)


LOGP = dict(X=fake(0), ldx=1000, f32=0, targets=fake(1), logp=fake(2), entropy=fake(3), lse=fake(4),
            top_logp=fake(5), top_ids=fake(6), rows=8, V=1000, top=4, ws=fake(7), bytes=1 << 20)
GRAD = dict(X=fake(0), ldx=1000, f32=0, targets=fake(1), lse=fake(4), entropy=fake(3),
            g_logp=fake(8), g_entropy=fake(9), g_lse=fake(10), dX=fake(11), lddx=1000, rows=8,
            V=1000)


def test_logprob_refusals(lib):
    for n in ("X", "targets", "logp", "entropy", "lse", "top_logp", "top_ids"):
        assert call(lib, "dd_logprobs_fwd", LOGP, **{n: None}) == NULL, n
    for kw in (dict(rows=0), dict(V=0), dict(top=-1), dict(top=65), dict(top=5, V=4), dict(ldx=999),
               dict(rows=(1 << 23) + 1), dict(rows=1 << 22, V=1 << 20, ldx=1 << 20),
               dict(V=(1 << 30) + 1, ldx=1 << 31)):
        assert call(lib, "dd_logprobs_fwd", LOGP, **kw) == SHAPE, kw
    for kw in (dict(X=fake(0, 1)), dict(X=fake(0, 2), f32=1), dict(targets=fake(1, 4)),
               dict(logp=fake(2, 2)), dict(entropy=fake(3, 1)), dict(lse=fake(4, 2)),
               dict(top_logp=fake(5, 2)), dict(top_ids=fake(6, 4))):
        assert call(lib, "dd_logprobs_fwd", LOGP, **kw) == ALIGN, kw
    for kw in (dict(logp=fake(0, 4)), dict(lse=fake(3, 8)), dict(top_ids=fake(1)),
               dict(top_logp=fake(6))):
        assert call(lib, "dd_logprobs_fwd", LOGP, **kw) == ALIAS, kw
    need = lib.dd_logprobs_workspace_bytes(8, 150432, 4)
    assert need > 0 and lib.dd_logprobs_workspace_bytes(8, 0, 0) == 0
    wide = dict(LOGP, V=150432, ldx=150432)
    assert call(lib, "dd_logprobs_fwd", wide, ws=None) == WORKSPACE
    assert call(lib, "dd_logprobs_fwd", wide, bytes=need - 1) == WORKSPACE
    assert call(lib, "dd_logprobs_fwd", wide, ws=fake(7, 4)) == ALIGN
    assert call(lib, "dd_logprobs_fwd", wide, ws=fake(0, 64)) == ALIAS


def test_logprob_gradient_refusals(lib):
    for n in ("X", "targets", "lse", "entropy", "dX"):
        assert call(lib, "dd_logprobs_bwd", GRAD, **{n: None}) == NULL, n
    for kw in (dict(rows=0), dict(V=0), dict(ldx=999), dict(lddx=999),
               dict(V=(1 << 30) + 1, ldx=1 << 31, lddx=1 << 31)):
        assert call(lib, "dd_logprobs_bwd", GRAD, **kw) == SHAPE, kw
    for kw in (dict(X=fake(0, 1)), dict(dX=fake(11, 2), f32=1), dict(targets=fake(1, 4)),
               dict(lse=fake(4, 2)), dict(g_logp=fake(8, 1)), dict(g_entropy=fake(9, 2)),
               dict(g_lse=fake(10, 3))):
        assert call(lib, "dd_logprobs_bwd", GRAD, **kw) == ALIGN, kw
    for kw in (dict(dX=fake(0, 2)), dict(dX=fake(0), lddx=1008), dict(dX=fake(1)), dict(dX=fake(8))):
        assert call(lib, "dd_logprobs_bwd", GRAD, **kw) == ALIAS, kw


def test_wrappers_refuse_what_is_not_on_a_gpu():
    q = torch.zeros(4, 2, 64, dtype=torch.bfloat16)
    pages = torch.zeros(3, 2, 16, 64, dtype=torch.bfloat16)
    ints = torch.zeros(2, dtype=torch.int32)
    table = torch.zeros(2, 2, dtype=torch.int32)
    with pytest.raises(ValueError, match="GPU"):
        cache.cache_attention(q, pages, pages, table, ints, ints)
    with pytest.raises(ValueError, match="GPU"):
        cache.cache_append(q, q, q, pages, pages, table, ints, ints)
    with pytest.raises(ValueError, match="GPU"):
        cache.cache_evict(pages, pages, table, ints, None, None, ints, 4)
    with pytest.raises(ValueError, match="3-D"):
        cache.cache_attention(q[0], pages, pages, table, ints, ints)
    with pytest.raises(ValueError, match="GPU"):
        lp.logprobs(torch.zeros(2, 5), torch.zeros(2, dtype=torch.int64))
    with pytest.raises(ValueError, match="2-D"):
        lp.logprobs(torch.zeros(5), torch.zeros(2, dtype=torch.int64))


def test_paged_cache_bookkeeping():
    """Pages and lengths of a cache on the CPU (no kernel runs)."""
    c = cache.PagedCache(2, 1, 64, 100, page=16, weights=True, device="cpu")
    assert c.per == 7 and len(c.free) == 14
    c._reserve([17, 0])
    assert [len(o) for o in c.owned] == [2, 0] and len(c.free) == 12
    assert c.table[0, :2].tolist() == c.owned[0] and (c.table[0, 2:] == -1).all()
    c.lengths = [17, 0]
    with pytest.raises(RuntimeError, match="slots"):
        c._reserve([96, 0])
    small = cache.PagedCache(2, 1, 64, 100, page=16, pages=3, device="cpu")
    with pytest.raises(RuntimeError, match="pages"):
        small._reserve([40, 20])
    assert small.owned == [[], []] and len(small.free) == 3
    c.clear(0)
    assert c.owned == [[], []] and len(c.free) == 14 and (c.table == -1).all()
    cache.check_cache(c.table, c.lens, pages=14, page=16)
    with pytest.raises(ValueError, match="weights=True"):
        small.evict(10)
    with pytest.raises(ValueError):
        c.extend(torch.zeros(2, 1, 64), None, None, [1])
    with pytest.raises(ValueError):
        c.extend(torch.zeros(2, 1, 64), None, None, [2, 1])


def test_block_extend_wants_as_many_rows_as_new_tokens():
    from paper_2405_13226_amd.layer import OpenLMBlock
    block = OpenLMBlock(d=512, H=8, hidden=256, device="cpu")
    c = cache.PagedCache(2, 8, 64, 64, page=16, device="cpu")
    x = torch.zeros(3, 512, dtype=torch.bfloat16)
    for rows, news in ((3, [10, 0]), (3, [2, 2]), (3, [1, 1]), (3, [3]), (3, [4, -1]), (3, [1, 1, 1]),
                       (0, [1, 0]), (0, [1, -1]), (0, [0])):
        with pytest.raises(ValueError, match="new tokens"):
            block.extend(x[:rows], c, news)
        assert c.lengths == [0, 0] and c.owned == [[], []] and not c.lens.any()
    assert block.extend(x[:0], c, [0, 0]).shape == (0, 512)


def test_the_cache_hands_over_the_chunks_rows_only(monkeypatch):
    """Rows behind the chunk's last are no tokens: the operators, whose plans go
    by the number of rows, get the chunk's; results have all rows, those behind
    as they were."""
    seen = []

    def append(q, k, v, *_, **kw):
        seen.append([t.shape[0] for t in (q, k, v)])
        return q

    def attention(q, *_, out=None, lse=None, **kw):
        seen.append([t.shape[0] for t in (q, out, lse)])
        out.fill_(1)
        lse.fill_(1)
        return out, lse
    monkeypatch.setattr(cache, "cache_append", append)
    monkeypatch.setattr(cache, "cache_attention", attention)
    c = cache.PagedCache(2, 2, 64, 64, page=16, device="cpu")
    q, k, v = (torch.zeros(256, h, 64, dtype=torch.bfloat16) for h in (4, 2, 2))
    out, lse = torch.full_like(q, 7.0), torch.full((256, 4), 7.0)
    o, z = c.extend(q, k, v, [2, 1], out=out, lse=lse)
    assert seen == [[3, 3, 3], [3, 3, 3]] and c.lens.tolist() == [2, 1] == c.lengths
    assert o is out and z is lse
    assert (out[:3] == 1).all() and (out[3:] == 7).all() and (lse[3:] == 7).all()
    o, z = c.extend(q, k, v, [0, 5])
    assert seen[2:] == [[5, 5, 5], [5, 5, 5]] and o.shape == q.shape and z.shape == (256, 4)
    state = [list(c.lengths), [list(p) for p in c.owned], list(c.free)]
    for bad in (dict(k=k[:200]), dict(v=v[:5]), dict(out=out[:3], lse=lse), dict(out=out),
                dict(out=out, lse=lse[:3]), dict(out=out, lse=lse.double())):
        args = dict(dict(k=k, v=v), **bad)
        with pytest.raises(ValueError):
            c.extend(q, args.pop("k"), args.pop("v"), [30, 1], **args)
        assert state == [c.lengths, c.owned, c.free], bad


def test_workspace_sizes_that_are_remembered_are_bounded():
    for rows in range(1, 3000):
        cache._bytes("dd_logprobs_workspace_bytes", rows, 100, 0)
    assert cache._bytes.cache_info().currsize <= 1024


def test_scores_are_not_kept_for_more_slots_than_a_launch_has_blocks(lib):
    """A block of 256 threads turns the scores of 1024 slots into weights, and a
    launch ends at 2^32 threads (weights of 68 GB); half of them are left to the
    joins.  On either side of the bound: the workspace with and without weights."""
    for per, kept in ((1 << 12, True), (1 << 14, False)):
        sizes = (1, 65535, 1, 1, 64, 16, per)
        more = lib.dd_cache_attn_workspace_bytes(*sizes, 1) - \
            lib.dd_cache_attn_workspace_bytes(*sizes, 0)
        assert more == (4 * 16 * per if kept else 0)


def test_the_cache_compares_its_rows_first():
    """What is no tensor of q's rows is refused before pages change hands."""
    c = cache.PagedCache(1, 2, 64, 64, page=16, device="cpu")
    q = torch.zeros(8, 2, 64, dtype=torch.bfloat16)
    for k, v in ((None, q), (q, None), (q[0, 0, 0], q), (q, q[:3])):
        with pytest.raises(ValueError):
            c.extend(q, k, v, [5])
    assert c.owned == [[]] and len(c.free) == 4

"""GPU parity of the paged cache (append, attention with slot weights,
eviction) against its float64 definitions.  Tolerances: tests/cache_oracle.py;
rows that are only moved, positions and lengths are exact."""
import random

import pytest
import torch

import paper_2405_13226_amd as dd

import cache_oracle as O
from parity import log

pytestmark = pytest.mark.gpu
BASE = 1e5

# lens, news, H, Hkv, D, page, tail: both kernels (few rows and many), with and
# without a split over workgroups; sequences without tokens, without slots,
# chunks of one token; tiles that end inside a page, pages inside a tile; heads
# of their own and shared by 2, 3, 4, 7 and 16
CASES = [
    ([0], [1], 1, 1, 64, 16, 0),
    ([0], [1], 3, 3, 128, 64, 3),
    ([63], [1], 2, 2, 128, 64, 0),
    ([64], [1], 2, 1, 64, 64, 0),
    ([1000], [1], 12, 12, 64, 64, 0),
    ([1000, 1, 0, 517], [1, 1, 1, 0], 16, 4, 128, 16, 2),
    ([300, 0, 40, 31], [5, 7, 0, 1], 6, 2, 64, 32, 1),
    ([4095], [1], 8, 8, 128, 128, 0),
    ([2047, 777], [3, 2], 14, 2, 128, 64, 0),
    ([1500], [17], 16, 1, 64, 16, 0),
    ([0], [129], 2, 2, 128, 64, 0),
    ([0, 5], [200, 64], 2, 1, 64, 16, 5),
    ([513, 0, 100], [130, 0, 257], 4, 4, 128, 32, 0),
    ([2500], [65], 3, 1, 64, 64, 0),
    ([700, 64], [66, 190], 4, 2, 64, 1024, 7),
    ([31, 32, 33, 127, 128, 129], [33, 97, 95, 1, 128, 127], 2, 2, 64, 16, 0),
    # few rows on the average, many in one sequence; scores kept and not
    ([50] * 15 + [300], [1] * 15 + [100], 1, 1, 64, 16, 0),
    ([2000] + [5] * 11, [75] + [1] * 11, 2, 2, 128, 32, 0),
    ([300, 20], [9, 9], 2, 2, 64, 16, 3),
    # one part per head, several; scores kept and not
    ([3000, 200, 0], [1, 2, 1], 4, 2, 128, 32, 0),
    ([5000, 17], [1, 1], 4, 4, 64, 16, 1),
    ([6000], [20], 1, 1, 64, 64, 0),
    ([2500], [31], 1, 1, 128, 16, 2),
    # many rows of D = 64, long sequences and short: two and more parts
    ([4500, 10, 2000], [60, 45, 1], 1, 1, 64, 64, 1),
    ([6500], [300], 4, 1, 64, 16, 0),
    # around the most rows that count as few, one part and several
    ([900, 40], [16, 16], 1, 1, 128, 32, 0),
    ([900, 40], [17, 16], 1, 1, 128, 32, 0),
    ([3100, 40], [24, 24], 1, 1, 64, 32, 0),
    ([3100, 40], [24, 25], 1, 1, 64, 32, 0),
    ([9000, 100, 7000], [1, 2, 1], 8, 2, 128, 64, 0),
]


def close(got, ref, tol, what):
    got = got.double().cpu()
    assert torch.isfinite(got).all(), what
    off = (got - ref).abs() - tol
    assert (off <= 0).all(), (what, float(off.max()), float((got - ref).abs().max()))


def run(x, dev, **kw):
    t = x.to(dev)
    return t, dd.cache_attention(t["q"], t["k"], t["v"], t["table"], t["lens_t"], t["cu"], **kw)


def check(x, dev):
    """The batch through the attention, with weights, against the oracle; rows
    behind the chunk and slots behind the last keep what they held."""
    n = sum(x.news)
    (o, lse, w), (to, tl, tw) = O.attention(x)
    out = torch.full((x.T, x.H, x.D), 7.0, dtype=torch.bfloat16, device=dev)
    z = torch.full((x.T, x.H), 7.0, device=dev)
    got_w = torch.full(x.w.shape, 3.0, device=dev)
    t = x.to(dev)
    kw = dict(weights=t["w"], weights_out=got_w, out=out, lse=z)
    dd.cache_attention(t["q"], t["k"], t["v"], t["table"], t["lens_t"], t["cu"], **kw)
    close(out[:n], o[:n], to[:n], "o")
    close(z[:n], lse[:n], tl[:n], "lse")
    assert (out[n:] == 7).all() and (z[n:] == 7).all()
    assert torch.equal(t["w"].cpu(), x.w)
    for b in range(x.B):
        m = x.lens[b] + x.news[b]
        close(got_w[b, :, :m], w[b, :, :m], tw[b, :, :m], "weights")
        assert (got_w[b, :, m:] == 3).all()
    # without weights, and with them in place: the same results
    _, (o2, z2) = run(x, dev)
    assert torch.equal(o2[:n], out[:n]) and torch.equal(z2[:n], z[:n])
    wi = t["w"].clone()
    dd.cache_attention(t["q"], t["k"], t["v"], t["table"], t["lens_t"], t["cu"], weights=wi)
    for b in range(x.B):
        m = x.lens[b] + x.news[b]
        assert torch.equal(wi[b, :, :m], got_w[b, :, :m])
        assert torch.equal(wi[b, :, m:].cpu(), x.w[b, :, m:])


@pytest.mark.parametrize("case", CASES, ids=lambda c: "-".join(map(str, c)).replace(" ", ""))
def test_attention(cuda, case):
    lens, news, H, Hkv, D, page, tail = case
    log(f"cache attention {case}")
    check(O.Batch(lens, news, H, Hkv, D, page, seed=sum(lens) + sum(news), tail=tail), cuda)


@pytest.mark.parametrize("seed", range(12))
def test_attention_of_random_batches(cuda, seed):
    g = random.Random(seed)
    H, Hkv = g.choice([(1, 1), (2, 1), (3, 3), (6, 2), (8, 8), (10, 2), (8, 1)])
    B = g.choice([1, 2, 3, 9])
    top = g.choice([1, 1, 4, 40, 150])
    lens = [g.choice([0, 1, g.randint(0, 700)]) for _ in range(B)]
    news = [g.randint(0 if B > 1 else 1, top) for _ in range(B)]
    news[0] = max(news[0], 1)
    case = (lens, news, H, Hkv, g.choice([64, 128]), g.choice([16, 32, 64, 128]), g.choice([0, 5]))
    log(f"cache attention {case}")
    check(O.Batch(*case[:6], seed=seed, tail=case[6]), cuda)


@pytest.mark.parametrize("D", [64, 128])
def test_attention_of_large_scores(cuda, D):
    log(f"cache attention, large scores, D={D}")
    check(O.Batch([400, 90], [3, 150], 4, 2, D, 16, seed=D, scale=8.0), cuda)


@pytest.mark.parametrize("news", [[1, 1, 1], [150, 40, 129]])
@pytest.mark.parametrize("D", [64, 128])
def test_what_a_row_may_not_see_leaves_no_trace(cuda, news, D):
    """Slots behind the last, other pages and later tokens hold NaN, infinities
    and the largest values: results are those of a cache of zeros there."""
    log(f"cache attention, bad values in hidden slots, {news} D={D}")
    x = O.Batch([70, 0, 200], news, 4, 2, D, 16, seed=5)
    bad = torch.tensor([float("nan"), float("inf"), float("-inf"), 3.3e38]).to(torch.bfloat16)
    clean, dirty = (O.Batch([70, 0, 200], news, 4, 2, D, 16, seed=5) for _ in range(2))
    for y, fill in ((clean, None), (dirty, bad)):
        for pages in (y.k, y.v):
            hidden = torch.ones(pages.shape[0], y.page, dtype=torch.bool)
            for b in range(y.B):
                for j in range(y.lens[b] + y.news[b]):
                    hidden[y.table[b, j // y.page], j % y.page] = False
            p, r = torch.nonzero(hidden, as_tuple=True)
            pages[p, :, r] = 0 if fill is None else \
                fill[torch.arange(p.numel()) % 4][:, None, None].expand(-1, y.Hkv, y.D)
    _, (o, z) = run(clean, cuda)
    _, (o2, z2) = run(dirty, cuda)
    assert torch.isfinite(o).all() and torch.equal(o, o2) and torch.equal(z, z2)
    check(clean, cuda)
    # the last token's own key and value: only its row shows it
    for which in ("k", "v"):
        for f in range(3):
            y = O.Batch([70, 0, 200], news, 4, 2, D, 16, seed=5)
            at = y.lens[2] + y.news[2] - 1
            getattr(y, which)[y.table[2, at // 16], :, at % 16] = bad[f]
            _, (o, z) = run(y, cuda)
            last = y.T - 1
            (ref, zr, _), (to, tl, _) = O.attention(x)
            close(o[:last], ref[:last], to[:last], "earlier rows")
            close(z[:last], zr[:last], tl[:last], "earlier rows' lse")
            if which == "v":
                assert not torch.isfinite(o[last]).any()
                close(z[last:], zr[last:], tl[last:], "lse")


def test_values_not_finite_in_sight_reach_their_rows(cuda):
    """An infinite value in a slot that some rows see and others do not: the
    rows that see it are infinite in that element, the others exact."""
    log("cache attention, infinite values in sight")
    for news, j, c in [([40], 20, 7), ([200], 101, 7), ([1], 30, 7)] + \
            [([2], 31, c) for c in (0, 13, 32, 63)] + [([40], 30 + c // 2, c) for c in range(0, 64, 5)] + \
            [([100], 30 + c, c) for c in range(0, 64, 3)]:
        x = O.Batch([30], news, 2, 2, 64, 16, seed=3)
        (ref, _, _), (to, _, _) = O.attention(x)
        x.v[x.table[0, j // 16], :, j % 16, c] = float("inf")
        _, (o, _) = run(x, cuda)
        sees = torch.arange(news[0]) + 30 >= j
        o = o.cpu()
        assert (o[sees][:, :, c] == float("inf")).all()
        keep = torch.ones(news[0], 2, 64, dtype=torch.bool)
        keep[sees, :, c] = False
        assert ((o.double() - ref).abs() <= to)[keep].all()


def test_queries_as_columns_and_other_streams(cuda):
    log("cache attention, strided queries, another stream")
    x = O.Batch([100, 20], [3, 40], 4, 4, 64, 32, seed=9)
    t, (o, z) = run(x, cuda)
    wide = torch.zeros(x.T, 3 * 4 * 64, dtype=torch.bfloat16, device=cuda)
    wide[:, 256:512] = t["q"].view(x.T, -1)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        o2, z2 = dd.cache_attention(wide[:, 256:512].view(x.T, 4, 64), t["k"], t["v"], t["table"],
                                    t["lens_t"], t["cu"])
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(o, o2) and torch.equal(z, z2)


def test_attention_equals_the_training_forward(cuda):
    """A whole sequence as one chunk and as several: the causal forward's
    results, to the tolerance of the two."""
    log("cache attention against forward")
    q, k, v = (torch.randn(1, 700, 4, 128, device=cuda, dtype=torch.bfloat16) for _ in range(3))
    o, lse = dd.forward(q, k, v)
    for cuts in ([700], [1, 299, 400], [64] * 10 + [60]):
        cache = dd.PagedCache(1, 4, 128, 704, page=32, device=cuda)
        parts, at = [], 0
        for n in cuts:
            parts.append(cache.extend(*(t[0, at:at + n] for t in (q, k, v)), [n]))
            at += n
        got, z = (torch.cat(p) for p in zip(*parts))
        # both are within 2^-8 (|o| + sum p |v|) of the exact value; sum p |v| < max |v|
        tol = 2 * 2.0 ** -8 * (o.abs() + v.abs().amax()).float()
        assert ((got.float() - o[0].float()).abs() <= tol[0]).all()
        assert float((got.float() - o[0].float()).norm() / o.float().norm()) < 2 ** -7
        assert float((z - lse[0]).abs().max()) < 1e-4


@pytest.mark.parametrize("rope", [None, BASE])
@pytest.mark.parametrize("D,page", [(64, 16), (128, 64)])
def test_append(cuda, D, page, rope):
    log(f"append D={D} page={page} rope={rope}")
    x = O.Batch([40, 0, 7, 100], [9, 3, 0, 1], 6, 2, D, page, seed=D, tail=4)
    T, Hkv = x.T, 2
    n = sum(x.news)
    kv = torch.randn(T, 2, Hkv, D).to(torch.bfloat16)
    start = torch.tensor([50, 0, 9, 16000], dtype=torch.int32)
    t = x.to(cuda)
    kvd = kv.to(cuda)
    pos_out = torch.full((x.B, Hkv, x.slots), -5, dtype=torch.int32, device=cuda)
    out = torch.full((T, 6, D), 7.0, dtype=torch.bfloat16, device=cuda) if rope else None
    q = dd.cache_append(t["q"], kvd[:, 0], kvd[:, 1], t["k"], t["v"], t["table"], t["lens_t"],
                        t["cu"], rope_base=rope, start=start.to(cuda), positions=pos_out, out=out)
    pos = torch.cat([int(s) + torch.arange(m) for s, m in zip(start, x.news)])
    if rope:
        # bit-identical to the rotation of a row of consecutive positions
        full = torch.zeros(1, 16064, 6, D, dtype=torch.bfloat16, device=cuda)
        fullk = torch.zeros(1, 16064, Hkv, D, dtype=torch.bfloat16, device=cuda)
        for i, p in enumerate(pos.tolist()):  # tokens of one position: one after the other
            full[0, p], fullk[0, p] = t["q"][i], kvd[i, 0]
            want = dd.rope(full, rope)[0, p]
            assert torch.equal(q[i], want)
            kv[i, 0] = dd.rope(fullk, rope)[0, p].cpu()
        assert (q[n:] == 7).all()
        ref = O.rotate(x.q[:n], pos, rope)
        # one rounding to bf16, sine and cosine to 2^-21
        assert ((q[:n].double().cpu() - ref).abs() <= O.HB * ref.abs() + 2.0 ** -19 * 6).all()
    else:
        assert q is t["q"]
    want_k, want_v, want_p = x.k.clone(), x.v.clone(), torch.full((x.B, Hkv, x.slots), -5)
    i = 0
    for b in range(x.B):
        for j in range(x.lens[b], x.lens[b] + x.news[b]):
            p = int(x.table[b, j // page])
            want_k[p, :, j % page], want_v[p, :, j % page] = kv[i, 0], kv[i, 1]
            want_p[b, :, j] = pos[i]
            i += 1
    assert torch.equal(t["k"].cpu(), want_k) and torch.equal(t["v"].cpu(), want_v)
    assert torch.equal(pos_out.cpu(), want_p.int())


def test_append_without_a_slot_or_a_page_writes_nothing(cuda):
    log("append without slots")
    x = O.Batch([30, 5], [4, 4], 2, 2, 64, 16, seed=1, spare=0)
    t = x.to(cuda)
    kv = torch.ones(x.T, 2, 64, dtype=torch.bfloat16, device=cuda)
    table = t["table"].clone()
    table[1, 0] = x.pages  # the cache has no such page
    dd.cache_append(None, kv, kv, t["k"], t["v"], table,
                    torch.tensor([x.slots - 2, 5], dtype=torch.int32, device=cuda), t["cu"])
    want = x.k.clone()
    for j in (x.slots - 2, x.slots - 1):
        p = int(x.table[0, j // 16])
        want[p, :, j % 16] = 1
    assert torch.equal(t["k"].cpu(), want)


def evict_case(cuda, lens, w, pos, seen, budget, recent, D=64, page=16, in_place=False):
    B, Hkv, slots = w.shape
    per = slots // page
    g = torch.Generator().manual_seed(slots)
    table = torch.randperm(B * per, generator=g).int().view(B, per)
    k, v = (torch.randn(B * per, Hkv, page, D, generator=g).to(torch.bfloat16) for _ in range(2))
    d = [t.to(cuda) for t in (k, v, table, lens, w, pos, seen)]
    out = (d[4], d[5], d[3]) if in_place else (torch.full_like(d[4], 9.0), torch.full_like(d[5], 9),
                                               torch.full_like(d[3], 9))
    res = dd.cache_evict(*d, budget, recent, out=out)
    want = [t.clone() for t in (k, v, w, pos)]
    for (b, h), pairs in O.evict(lens, w, pos, seen, budget, recent).items():
        for to, src in pairs:
            pt, ps = int(table[b, to // page]), int(table[b, src // page])
            want[0][pt, h, to % page] = k[ps, h, src % page]
            want[1][pt, h, to % page] = v[ps, h, src % page]
            want[2][b, h, to], want[3][b, h, to] = w[b, h, src], pos[b, h, src]
    left = torch.clamp(lens, max=budget)
    assert torch.equal(res[2].cpu(), left)
    assert torch.equal(d[0].cpu(), want[0]) and torch.equal(d[1].cpu(), want[1])
    for b in range(B):
        n = int(left[b])
        assert torch.equal(res[0][b, :, :n].cpu().view(torch.int32),
                           want[2][b, :, :n].view(torch.int32))
        assert torch.equal(res[1][b, :, :n].cpu(), want[3][b, :, :n])
        # behind the new lens: the inputs' up to the budget, then what was there
        rest = (w.clone(), pos.clone())
        if not in_place:
            rest[0][..., budget:], rest[1][..., budget:] = 9.0, 9
        assert torch.equal(res[0][b, :, n:].cpu().view(torch.int32),
                           rest[0][b, :, n:].view(torch.int32))
        assert torch.equal(res[1][b, :, n:].cpu(), rest[1][b, :, n:])


def evict_state(lens, Hkv, slots, seed, ties=False):
    g = torch.Generator().manual_seed(seed)
    B = len(lens)
    w = torch.exp(2 * torch.randn(B, Hkv, slots, generator=g))
    if ties:
        w = torch.randint(0, 4, w.shape, generator=g).float()
        w[w == 0] *= torch.where(torch.rand(int((w == 0).sum()), generator=g) < 0.5, -1.0, 1.0)
    pos = torch.cumsum(torch.randint(1, 4, w.shape, generator=g), dim=2).int()
    lens = torch.tensor(lens, dtype=torch.int32)
    last = [int(pos[b, :, int(n) - 1].max()) + 1 if n else 0 for b, n in enumerate(lens)]
    return lens, w, pos, torch.tensor(last, dtype=torch.int32)


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("ties", [False, True])
@pytest.mark.parametrize("lens,slots,budget,recent", [
    ([12000, 9000], 12016, 5000, 100), ([20000], 20000, 17000, 3),
    ([100, 7, 0, 64], 112, 40, 8), ([5], 16, 1, 0), ([5], 16, 1, 1), ([48, 47], 48, 47, 47),
    ([48], 48, 48, 3), ([3000, 2999], 3008, 1025, 300), ([2100], 2112, 2000, 0),
    ([1300, 1200], 1312, 64, 64)])
def test_evict(cuda, lens, slots, budget, recent, ties, in_place):
    log(f"evict {lens} of {slots} to {budget}, recent {recent}, ties {ties}")
    st = evict_state(lens, 3, slots, slots + budget, ties)
    evict_case(cuda, *st, budget, recent, in_place=in_place)


def test_evict_of_weights_out_of_the_ordinary(cuda):
    log("evict: NaN, infinities, negative weights, all equal, recent everywhere")
    lens, w, pos, seen = evict_state([500, 480], 2, 512, 3)
    w[0, 0, 10:200:7] = float("nan")
    w[0, 1, ::3] = float("inf")
    w[1, 0] = -w[1, 0]
    w[1, 0, 5] = float("-inf")
    w[1, 1] = 1.0
    evict_case(cuda, lens, w, pos, seen, 450, 16, D=128)
    w[0] = float("nan")
    pos[:] = 100  # every slot within the last positions
    seen[:] = 100
    evict_case(cuda, lens, w, pos, seen, 100, 1, D=128)
    seen[:] = -2 ** 31  # seen - recent leaves int32
    evict_case(cuda, lens, w, pos, seen, 100, 100, D=128)


def test_a_run_of_all(cuda):
    """Generation with eviction: chunks of a prompt, then single tokens; after
    each eviction the attention is the one over the slots that were kept."""
    log("cache: prompt, generation, eviction")
    H, Hkv, D, budget, recent = 4, 2, 64, 48, 16
    g = torch.Generator().manual_seed(0)
    cache = dd.PagedCache(2, Hkv, D, 160, page=16, weights=True, device=cuda)
    kept = [[{} for _ in range(Hkv)] for _ in range(2)]  # position -> (k, v, weight)
    for step in range(30):
        news = [50, 33] if step == 0 else [7, 0] if step == 1 else [1, 1]
        T = sum(news)
        q, k, v = (torch.randn(T, h, D, generator=g).to(torch.bfloat16) for h in (H, Hkv, Hkv))
        o, _ = cache.extend(q.to(cuda), k.to(cuda), v.to(cuda), news, rope_base=BASE)
        at = 0
        for b in range(2):
            seen = cache.tokens[b] - news[b]
            pos = seen + torch.arange(news[b])
            qr, kr = (O.rotate(t[at:at + news[b]], pos, BASE) for t in (q, k))
            qr, kr = (t.to(torch.bfloat16).double() for t in (qr, kr))
            for i in range(news[b]):
                for h in range(Hkv):
                    c = kept[b][h]
                    c[seen + i] = [kr[i, h], v[at + i, h].double(), 0.0]
                    ks, vs = (torch.stack([e[n] for e in c.values()]) for n in (0, 1))
                    for x in range(2):
                        p = torch.softmax(ks @ qr[i, 2 * h + x] / 8, dim=0)
                        # two roundings of 2^-8 and a rotated key's or query's other one
                        ref = p @ vs
                        tol = 0.02 * (p @ vs.abs()) + 0.01 * ref.abs()
                        assert ((o[at + i, 2 * h + x].double().cpu() - ref).abs() <= tol).all()
                        for e, y in zip(c.values(), p.tolist()):
                            e[2] += y
            at += news[b]
        if step % 10 == 9 or step == 1:
            cache.evict(budget, recent)
            # which slots stay is decided by the device's weights; they agree with
            # the ones summed here, and the recent ones are among them
            for b in range(2):
                n = cache.lengths[b]
                assert n <= budget and len(cache.owned[b]) == -(-n // 16)
                for h in range(Hkv):
                    pos = cache.positions[b, h, :n].tolist()
                    assert len(set(pos)) == n
                    want = cache.tokens[b] - 1
                    assert set(range(want - min(recent, n) + 1, want + 1)) <= set(pos)
                    got = cache.weights[b, h, :n].double().cpu()
                    ref = torch.tensor([kept[b][h][p][2] for p in pos])
                    assert ((got - ref).abs() <= 0.02 * ref + 1e-3).all()
                    gone = [e[2] for p, e in kept[b][h].items()
                            if p not in set(pos) and p < cache.tokens[b] - recent]
                    stay = [kept[b][h][p][2] for p in pos if p < cache.tokens[b] - recent]
                    if gone and stay:
                        assert max(gone) <= min(stay) * 1.02 + 1e-3
                    kept[b][h] = {p: kept[b][h][p] for p in pos}
    assert len(cache.free) == 20 - sum(len(o) for o in cache.owned)
    cache.clear(0)
    assert not cache.owned[0] and int(cache.lens[0]) == 0


def test_graph_of_a_token(cuda):
    """Append, attention with weights and eviction captured once and replayed
    with other contents, two graphs in turn, eager work between."""
    log("cache: graphs")
    H, D = 4, 64
    xs = [O.Batch([37, 150], [1, 1], H, 2, D, 16, seed=s) for s in (0, 1)]
    graphs = []
    for x in xs:
        t = x.to(cuda)
        t["kn"], t["vn"] = (torch.randn(2, 2, D, device=cuda).to(torch.bfloat16) for _ in range(2))
        t["pos"] = torch.zeros(2, 2, x.slots, dtype=torch.int32, device=cuda)
        t["start"] = t["lens_t"].clone()
        t["seen"] = t["lens_t"] + 1

        def step(t=t):
            q = dd.cache_append(t["q"], t["kn"], t["vn"], t["k"], t["v"], t["table"], t["lens_t"],
                                t["cu"], rope_base=BASE, start=t["start"], positions=t["pos"])
            w = torch.empty_like(t["w"])
            o, z = dd.cache_attention(q, t["k"], t["v"], t["table"], t["lens_t"], t["cu"],
                                      weights=t["w"], weights_out=w)
            after = t["lens_t"] + 1
            e = dd.cache_evict(t["k"], t["v"], t["table"], after, w, t["pos"], t["seen"], 30, 4)
            return o, z, *e
        first = [t["k"].clone(), t["v"].clone()]
        step()  # warm up
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            out = step()
        graphs.append((graph, out, t, first, step))
    for _ in range(3):
        for graph, out, t, first, step in graphs:
            t["q"].copy_(torch.randn_like(t["q"]))
            t["k"].copy_(first[0]), t["v"].copy_(first[1])
            want = [y.clone() for y in step()]
            kv = [t["k"].clone(), t["v"].clone()]
            t["k"].copy_(first[0]), t["v"].copy_(first[1])
            graph.replay()
            torch.cuda.synchronize()
            n = 30
            assert torch.equal(out[0], want[0]) and torch.equal(out[1], want[1])
            for b in range(2):
                assert torch.equal(out[2][b, :, :n], want[2][b, :, :n])
                assert torch.equal(out[3][b, :, :n], want[3][b, :, :n])
            assert torch.equal(out[4], want[4])
            assert torch.equal(t["k"], kv[0]) and torch.equal(t["v"], kv[1])


def test_block_extend(cuda):
    """The block on a whole row, and in chunks through a cache."""
    log("block: extend")
    from paper_2405_13226_amd.layer import OpenLMBlock
    block = OpenLMBlock(d=512, H=8, hidden=1024, device=cuda)
    x = torch.randn(1, 512, 512, device=cuda, dtype=torch.bfloat16)
    with torch.no_grad():
        y = block(x)[0].float()
    cache = dd.PagedCache(1, 8, 64, 512, device=cuda)
    parts, at = [], 0
    for n in (300, 1, 1, 64, 146):
        parts.append(block.extend(x[0, at:at + n], cache, [n]))
        at += n
    got = torch.cat(parts).float()
    assert cache.lengths == [512]
    # the two differ by roundings of the attention's output (2^-8 each) and what follows
    assert float((got - y).norm() / y.norm()) < 2.0 ** -7


def test_caches_past_32_bits(cuda):
    """Pages behind 2^32 bytes and 2^31 elements."""
    log("cache: offsets past 32 bits")
    pages, Hkv, page, D = 9000, 8, 256, 128  # 2.36e9 elements
    k = torch.zeros(pages, Hkv, page, D, dtype=torch.bfloat16, device=cuda)
    v = torch.zeros_like(k)
    x = O.Batch([600, 100], [1, 40], 8, 8, 128, 256, seed=2)
    order = torch.arange(pages - 1, pages - 1 - x.pages, -1)
    table = torch.where((x.table >= 0) & (x.table < x.pages),
                        order[x.table.clamp(0, x.pages - 1).long()].int(), x.table)
    k[order.to(cuda)], v[order.to(cuda)] = x.k.to(cuda), x.v.to(cuda)
    t, (o, z) = run(x, cuda)
    w, w2 = t["w"].clone(), t["w"].clone()
    dd.cache_attention(t["q"], t["k"], t["v"], t["table"], t["lens_t"], t["cu"], weights=w)
    o2, z2 = dd.cache_attention(t["q"], k, v, table.to(cuda), t["lens_t"], t["cu"], weights=w2)
    assert torch.equal(o, o2) and torch.equal(z, z2) and torch.equal(w, w2)
    new = torch.ones(x.T, 8, 128, dtype=torch.bfloat16, device=cuda)
    dd.cache_append(None, new, new, k, v, table.to(cuda), t["lens_t"], t["cu"])
    assert (k[order[x.table[0, 600 // 256].item()], :, 600 % 256] == 1).all()
    pos = torch.zeros(x.B, 8, x.slots, dtype=torch.int32, device=cuda)
    seen = torch.zeros(2, dtype=torch.int32, device=cuda)
    a = dd.cache_evict(t["k"], t["v"], t["table"], t["lens_t"], w, pos, seen, 50)
    b = dd.cache_evict(k, v, table.to(cuda), t["lens_t"], w, pos, seen, 50)
    assert torch.equal(a[0][..., :50], b[0][..., :50])
    ids = t["table"][:, 0].long()
    assert torch.equal(t["k"][ids, :, :50], k[order.to(cuda)[ids], :, :50])


def test_outputs_stay_inside_their_buffers(cuda):
    """Canaries around every output; T x H odd, ragged."""
    log("cache: guard bands")
    from test_gpu_guard import Guarded
    x = O.Batch([77, 5, 130], [1, 3, 2], 6, 2, 64, 16, seed=4)
    t = x.to(cuda)
    for news_form in (False, True):
        if news_form:
            x = O.Batch([77, 5, 130], [190, 3, 65], 3, 1, 128, 16, seed=4)
            t = x.to(cuda)
        o = Guarded((x.T, x.H, x.D), torch.bfloat16, cuda)
        z = Guarded((x.T, x.H), torch.float32, cuda)
        w = Guarded(x.w.shape, torch.float32, cuda)
        p = Guarded(x.w.shape, torch.int32, cuda)
        kp, vp = (Guarded(t["k"].shape, torch.bfloat16, cuda) for _ in range(2))
        kp.t.copy_(t["k"]), vp.t.copy_(t["v"])
        new = torch.ones(x.T, x.Hkv, x.D, dtype=torch.bfloat16, device=cuda)
        q = Guarded((x.T, x.H, x.D), torch.bfloat16, cuda)
        dd.cache_append(t["q"], new, new, kp.t, vp.t, t["table"], t["lens_t"], t["cu"], rope_base=BASE,
                        positions=p.t, out=q.t)
        dd.cache_attention(q.t, kp.t, vp.t, t["table"], t["lens_t"], t["cu"], weights=t["w"],
                           weights_out=w.t, out=o.t, lse=z.t)
        ln = Guarded((x.B,), torch.int32, cuda)
        dd.cache_evict(kp.t, vp.t, t["table"], t["lens_t"], t["w"], p.t.clone(), t["lens_t"], 40, 8,
                       out=(w.t, p.t, ln.t))
        torch.cuda.synchronize()
        for buf in (o, z, w, p, kp, vp, q, ln):
            assert buf.intact()


def test_empty_calls(cuda):
    log("cache: empty calls")
    x = O.Batch([10], [0], 2, 2, 64, 16)
    t = x.to(cuda)
    o, z = dd.cache_attention(t["q"], t["k"], t["v"], t["table"], t["lens_t"], t["cu"])
    assert o.shape == (0, 2, 64) and z.shape == (0, 2)
    dd.cache_append(t["q"], t["q"], t["q"], t["k"], t["v"], t["table"], t["lens_t"], t["cu"])
    assert torch.equal(t["k"].cpu(), x.k)
    cache = dd.PagedCache(2, 2, 64, 64, page=16, device=cuda)
    q = torch.zeros(3, 2, 64, dtype=torch.bfloat16, device=cuda)
    with pytest.raises(RuntimeError):
        cache.extend(torch.zeros(65, 2, 64, dtype=torch.bfloat16, device=cuda), q, q, [65, 0])
    assert cache.lengths == [0, 0] and len(cache.free) == 8


def test_malformed_contents_stay_inside(cuda):
    """Lengths, offsets and pages out of range: nothing outside the tensors is
    touched (results are unspecified)."""
    log("cache: malformed contents")
    from test_gpu_guard import Guarded
    x = O.Batch([77, 5], [1, 3], 4, 2, 64, 16, seed=4)
    for lens, cu, fill in (([10 ** 9, -5], [0, 1, 4], None), ([77, 5], [-7, 10 ** 9, -3], None),
                           ([77, 5], [0, 1, 4], 2 ** 31 - 1), ([77, 5], [0, 1, 4], -2 ** 31)):
        t = x.to(cuda)
        lens = torch.tensor(lens, dtype=torch.int32, device=cuda)
        cu = torch.tensor(cu, dtype=torch.int32, device=cuda)
        if fill is not None:
            t["table"].fill_(fill)
        kp, vp = (Guarded(t["k"].shape, torch.bfloat16, cuda) for _ in range(2))
        kp.t.copy_(t["k"]), vp.t.copy_(t["v"])
        w, p = Guarded(x.w.shape, torch.float32, cuda), Guarded(x.w.shape, torch.int32, cuda)
        o, z = Guarded((4, 4, 64), torch.bfloat16, cuda), Guarded((4, 4), torch.float32, cuda)
        new = torch.ones(4, 2, 64, dtype=torch.bfloat16, device=cuda)
        dd.cache_append(None, new, new, kp.t, vp.t, t["table"], lens, cu, rope_base=BASE,
                        positions=p.t)
        dd.cache_attention(t["q"], kp.t, vp.t, t["table"], lens, cu, weights=t["w"],
                           weights_out=w.t, out=o.t, lse=z.t)
        dd.cache_evict(kp.t, vp.t, t["table"], lens, t["w"], p.t.clone(), lens.clone(), 20, 4,
                       out=(w.t, p.t, lens))
        torch.cuda.synchronize()
        for buf in (kp, vp, w, p, o, z):
            assert buf.intact()


def test_rows_behind_the_chunk_do_not_change_the_plan(cuda):
    """The cache's results for a token each are bit for bit those without the
    rows of padding behind them."""
    log("cache: padding rows")
    g = torch.Generator().manual_seed(3)
    caches = [dd.PagedCache(2, 4, 128, 4096, page=16, weights=True, device=cuda) for _ in range(2)]
    for news in ([900, 400], [1, 1], [1, 0], [1, 1]):
        n = sum(news)
        q, k, v = (torch.randn(n, 4, 128, generator=g).to(torch.bfloat16).to(cuda) for _ in range(3))
        o, z = caches[0].extend(q, k, v, news, rope_base=BASE)
        wide = [torch.nn.functional.pad(t, (0, 0, 0, 0, 0, 256)) for t in (q, k, v)]
        out, lse = torch.full_like(wide[0], 7.0), torch.full((n + 256, 4), 7.0, device=cuda)
        caches[1].extend(*wide, news, rope_base=BASE, out=out, lse=lse)
        assert torch.equal(out[:n], o) and torch.equal(lse[:n], z)
        assert (out[n:] == 7).all() and (lse[n:] == 7).all()
        for b in range(2):
            m = caches[0].lengths[b]
            assert torch.equal(*(c.weights[b, :, :m] for c in caches))


def test_block_extend_of_several_sequences_with_weights(cuda):
    """Chunks of three sequences through a cache with weights: the block on each
    whole row; rows of padding leave nothing in the cache, and a token each takes
    the plan of its rows alone."""
    log("block: extend of several sequences")
    from paper_2405_13226_amd.layer import OpenLMBlock
    block = OpenLMBlock(d=512, H=8, hidden=1024, device=cuda)
    x = torch.randn(3, 256, 512, device=cuda, dtype=torch.bfloat16)
    with torch.no_grad():
        y = block(x).float()
    cache = dd.PagedCache(3, 8, 64, 512, page=16, weights=True, device=cuda)
    at, got = [0, 0, 0], torch.zeros_like(y)
    for news in ([200, 0, 3], [1, 1, 1], [1, 1, 1], [0, 150, 0], [54, 104, 251]):
        rows = torch.cat([x[b, a:a + n] for b, (a, n) in enumerate(zip(at, news))])
        out = block.extend(rows, cache, news).float()
        assert out.shape == rows.shape
        i = 0
        for b, n in enumerate(news):
            got[b, at[b]:at[b] + n] = out[i:i + n]
            i, at[b] = i + n, at[b] + n
        assert cache.lengths == at == cache.lens.tolist()
    assert at == [256, 256, 256]
    # the two differ by roundings of the attention's output (2^-8 each) and what follows
    assert float((got - y).norm() / y.norm()) < 2.0 ** -7
    # a token's probabilities add up to 1 a head, each sum within 1e-4 (see cache_oracle)
    total = cache.weights.double().sum(dim=2)
    assert ((total[:, :, None] - 256).abs() <= 256 * 1e-4).all()
    cache.evict(100, 20)
    block.extend(x[:, 0], cache, [1, 1, 1])
    assert cache.lengths == [101] * 3


def test_evict_without_slots_or_heads(cuda):
    """Nothing to thin out: the lengths that are left all the same."""
    log("evict: no slots, no heads")
    lens = torch.tensor([7, 0, 90], dtype=torch.int32, device=cuda)
    seen = torch.zeros_like(lens)
    for Hkv, per, want in ((0, 6, [7, 0, 40]), (2, 0, [0, 0, 0])):
        pages = torch.zeros(4, Hkv, 16, 64, dtype=torch.bfloat16, device=cuda)
        table = torch.zeros(3, per, dtype=torch.int32, device=cuda)
        w = torch.zeros(3, Hkv, per * 16, device=cuda)
        n = torch.full_like(lens, -9)
        out = dd.cache_evict(pages, pages.clone(), table, lens, w, w.int(), seen, 40, 3,
                             out=(w.clone(), w.int(), n))
        assert out[2] is n and n.tolist() == want
        out = dd.cache_evict(pages, pages.clone(), table, lens, w, w.int(), seen, 40, 3)
        assert out[2].tolist() == want


def test_append_refuses_a_base_that_fp32_does_not_hold(cuda):
    log("append: rope bases that leave fp32")
    x = O.Batch([3], [2], 2, 2, 64, 16)
    t = x.to(cuda)
    for base in (1e-50, 1e39, -1.0, 0.0, float("nan"), float("inf")):
        for q in (None, t["q"]):
            with pytest.raises((ValueError, dd.DDError)):
                dd.cache_append(q, t["q"], t["q"], t["k"], t["v"], t["table"], t["lens_t"], t["cu"],
                                rope_base=base)
    assert torch.equal(t["k"].cpu(), x.k)


# many rows over capacities from which a workgroup forms the weights of 256 slots:
# chunks across such a border, sequences shorter than a block and without slots
@pytest.mark.parametrize("H,Hkv,D,page,spare", [(8, 8, 64, 1024, 22), (16, 8, 128, 1024, 22),
                                                (8, 8, 128, 16, 1400), (32, 16, 64, 64, 175)])
def test_weights_of_large_capacities(cuda, H, Hkv, D, page, spare):
    log(f"cache attention, large capacity, {H} {Hkv} {D} page {page}")
    x = O.Batch([200, 0, 700], [100, 40, 70], H, Hkv, D, page, seed=D + page, spare=spare, tail=2)
    assert -(-x.slots // 256) * x.B * Hkv >= 2048
    check(x, cuda)


# few rows, short caches, more (sequence, key head) pairs than run at once: a
# part each, the usual waves; scores kept and not
@pytest.mark.parametrize("H,D", [(8, 64), (8, 128), (96, 64), (128, 128)])
def test_many_heads_of_short_caches(cuda, H, D):
    log(f"cache attention, 80 sequences of 8 key heads, {H} heads of {D}")
    g = random.Random(H)
    lens = [g.choice([0, 1, 15, 16, 33, 64, 100]) for _ in range(80)]
    news = [g.choice([0, 1, 1, 2]) for _ in lens]
    check(O.Batch(lens, news, H, 8, D, 16, seed=H, tail=1), cuda)


@pytest.mark.parametrize("ties", [False, True])
@pytest.mark.parametrize("budget", [300, 19700])
@pytest.mark.parametrize("D", [64, 128])
def test_evict_few_rows_of_long_sequences(cuda, D, budget, ties):
    """Beyond 16,384 slots, moved by the workgroup that selects them."""
    log(f"evict 20000 to {budget}, D {D}, ties {ties}")
    evict_case(cuda, *evict_state([20000, 18000, 5], 2, 20000, budget, ties), budget, 40, D=D)

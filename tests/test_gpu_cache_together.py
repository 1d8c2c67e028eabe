"""The paged cache's calls as a serving program makes them: two at once on
streams of their own, captured and replayed with many rows, over pages that
sequences share, under a batch of prompts and single tokens."""
import random

import pytest
import torch

import paper_2405_13226_amd as dd

import cache_oracle as O
from parity import log
from test_gpu_cache import check, close

pytestmark = pytest.mark.gpu

# scores kept and parts joined; parts alone; many rows with weights formed anew,
# in parts and not
SHAPES = [
    ([3000, 200, 0], [1, 2, 1], 4, 2, 128, 32),
    ([6000], [20], 1, 1, 64, 64),
    ([513, 0, 100], [130, 0, 257], 4, 4, 128, 32),
    ([4000, 31], [90, 400], 2, 1, 64, 16),
]


def batch(shape, seed):
    return O.Batch(*shape, seed=seed)


def step(t, n, w):
    """Attention with weights, the log probabilities of what it returns as
    logits, and an eviction."""
    o, z = dd.cache_attention(t["q"], t["k"], t["v"], t["table"], t["lens_t"], t["cu"],
                              weights=t["w"], weights_out=w)
    logits = o.reshape(o.shape[0], -1)
    out = dd.logprobs(logits, t["targets"], top=3)
    after = t["lens_t"] + (t["cu"][1:] - t["cu"][:-1])
    return (o, z, w, *out,
            *dd.cache_evict(t["k"], t["v"], t["table"], after, w, t["pos"], after, n, 4))


def state(x, dev):
    t = x.to(dev)
    t["targets"] = torch.arange(x.T, device=dev) % (x.H * x.D)
    t["pos"] = torch.arange(x.slots, dtype=torch.int32, device=dev).expand_as(t["w"]).contiguous()
    return t


def same(got, want, x, budget):
    """Slots behind a sequence's last are not compared: no call writes them."""
    for i, (a, b) in enumerate(zip(got, want)):
        if i in (2, len(want) - 3, len(want) - 2):
            for s in range(x.B):
                n = x.lens[s] + x.news[s]
                n = n if i == 2 else min(n, budget)
                assert torch.equal(a[s, :, :n], b[s, :, :n]), i
        else:
            assert torch.equal(a, b), i


@pytest.mark.parametrize("first,second", [(0, 1), (0, 2), (2, 3)])
def test_two_streams_at_once(cuda, first, second):
    log(f"cache: two streams, shapes {first} and {second}")
    xs = [batch(SHAPES[first], 1), batch(SHAPES[second], 2)]
    ts, kv, want = [], [], []
    for x in xs:
        t = state(x, cuda)
        ts.append(t)
        kv.append((t["k"].clone(), t["v"].clone()))
        out = step(t, 64, torch.zeros_like(t["w"]))
        want.append((out, t["k"].clone(), t["v"].clone()))
    for _ in range(3):
        for t, (k, v) in zip(ts, kv):
            t["k"].copy_(k), t["v"].copy_(v)
        ws = [torch.zeros_like(t["w"]) for t in ts]
        sides, got = [torch.cuda.Stream() for _ in ts], []
        torch.cuda.synchronize()
        for side, t, w in zip(sides, ts, ws):
            with torch.cuda.stream(side):
                got.append(step(t, 64, w))
        torch.cuda.synchronize()
        for x, t, out, (ref, k, v) in zip(xs, ts, got, want):
            same(out, ref, x, 64)
            assert torch.equal(t["k"], k) and torch.equal(t["v"], v)


@pytest.mark.parametrize("shape", range(len(SHAPES)))
def test_graph(cuda, shape):
    log(f"cache: graph of shape {shape}")
    x = batch(SHAPES[shape], 5)
    t = state(x, cuda)
    kv = [t["k"].clone(), t["v"].clone()]
    w = torch.zeros_like(t["w"])
    step(t, 64, w)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step(t, 64, w)
    for _ in range(3):
        t["q"].copy_(torch.randn_like(t["q"]))
        t["k"].copy_(kv[0]), t["v"].copy_(kv[1])
        want = [y.clone() for y in step(t, 64, torch.zeros_like(t["w"]))]
        after = [t["k"].clone(), t["v"].clone()]
        t["k"].copy_(kv[0]), t["v"].copy_(kv[1])
        graph.replay()
        torch.cuda.synchronize()
        same(out, want, x, 64)
        assert torch.equal(t["k"], after[0]) and torch.equal(t["v"], after[1])


@pytest.mark.parametrize("news", [[2, 2, 2], [2, 140, 33]])
def test_attention_over_shared_pages(cuda, news):
    """Sequences that begin with the same pages (attention reads them only)."""
    log(f"cache: shared pages, {news}")
    x = O.Batch([200, 200, 150], news, 4, 2, 64, 32, seed=3)
    x.table[1, :4] = x.table[0, :4]
    x.table[2, :4] = x.table[0, :4]
    n = sum(news)
    (o, lse, w), (to, tl, tw) = O.attention(x)
    t = x.to(cuda)
    got, z = dd.cache_attention(t["q"], t["k"], t["v"], t["table"], t["lens_t"], t["cu"],
                                weights=t["w"])
    close(got[:n], o[:n], to[:n], "o")
    close(z[:n], lse[:n], tl[:n], "lse")
    for b in range(x.B):
        m = x.lens[b] + x.news[b]
        close(t["w"][b, :, :m], w[b, :, :m], tw[b, :, :m], "weights")


@pytest.mark.parametrize("H,Hkv,D", [(4, 2, 128), (4, 4, 64)])
def test_prompts_among_single_tokens(cuda, H, Hkv, D):
    """A batch in which one sequence brings a prompt and the others a token: the
    results of the single tokens are those of a call of their own, to the
    tolerance of both."""
    log(f"cache: a prompt among tokens, {H} {Hkv} {D}")
    lens, news = [700, 0, 1500, 64, 1], [1, 300, 1, 1, 1]
    x = O.Batch(lens, news, H, Hkv, D, 16, seed=8)
    n = sum(news)
    (o, lse, _), (to, tl, _) = O.attention(x)
    t = x.to(cuda)
    got, z = dd.cache_attention(t["q"], t["k"], t["v"], t["table"], t["lens_t"], t["cu"])
    close(got[:n], o[:n], to[:n], "o")
    close(z[:n], lse[:n], tl[:n], "lse")
    for b, at in ((0, 0), (2, 301), (3, 302), (4, 303)):
        cu = torch.tensor([0, 1], dtype=torch.int32, device=cuda)
        one, z1 = dd.cache_attention(t["q"][at:at + 1], t["k"], t["v"], t["table"][b:b + 1],
                                     t["lens_t"][b:b + 1], cu)
        close(one, o[at:at + 1], to[at:at + 1], "o of its own")
        close(z1, lse[at:at + 1], tl[at:at + 1], "lse of its own")


@pytest.mark.parametrize("most", [1, 40])
@pytest.mark.parametrize("D", [64, 128])
def test_many_sequences(cuda, D, most):
    """More sequences than a wave has lanes, many of them without new tokens or
    without slots."""
    log(f"cache: 150 sequences, D {D}, up to {most} new tokens")
    rng = random.Random(D + most)
    lens = [rng.choice([0, 1, 15, 16, 17, 40, 130]) for _ in range(150)]
    news = [rng.choice([0, 1, rng.randint(1, most)]) for _ in lens]
    check(O.Batch(lens, news, 2, 1, D, 16, seed=most, tail=3), cuda)


def test_empty_batch(cuda):
    cache = dd.PagedCache(0, 2, 64, 64, page=16, device=cuda, weights=True)
    q = torch.zeros(0, 2, 64, dtype=torch.bfloat16, device=cuda)
    o, z = cache.extend(q, q, q, [])
    assert o.shape == (0, 2, 64) and z.shape == (0, 2)
    cache.evict(4)

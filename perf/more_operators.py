"""What a trained model answers with and learns from: a paged cache of keys
and values, the attention that reads it, eviction from it, and the log
probabilities of given tokens with their gradient.

    append     rotary embedding of a ragged chunk's q and k at their positions,
               k and v written into the cache's pages
    attend     causal attention of the chunk's queries over the cache
    track      the same, and the attention weight of each cached slot added to
               what it has so far
    evict      the slots with the most weight stay, the survivors behind the
               budget move into the holes before it
    logprob    log probability of given tokens, entropy, log of the sum of
               exponentials, and the most likely alternatives
    loss       the same without alternatives, and the gradient of the logits

    listed()                 the named cases
    draw(rng)                one more case of the same ranges
    prepare(case, seed)      what the program holds before the call
    run(state)               one pass; returns every output whole
    work(case)               bytes and flops that the pass cannot do without
    exact(case, seed)        the same outputs in 64 bits

`own` says whether run() calls this package or computes the plain form.

A cache holds keys and values as pages [pages, kv heads, page, D] of bf16;
`table` [B, pages per sequence] names the pages of each sequence in order.
Sequence b has lens[b] slots in use before the call and gets the rows
cu_new[b] .. cu_new[b + 1] of the chunk.
"""
from __future__ import annotations

import math
import random

import torch

own = False

DEVICE = "cuda"
ROPE_BASE = 100000.0


def listed():
    return [
        # generation of one sequence: one token's keys and values; latency alone
        dict(kind="append", B=1, new=1, ctx=1000, H=16, Hkv=16, D=128, page=64, name="append_one"),
        # a long prompt batch enters the cache in one chunk
        dict(kind="append", B=8, new=4096, ctx=4000, H=16, Hkv=16, D=128, page=64,
             name="append_chunk"),
        # generation of one sequence with the smallest model; latency alone
        dict(kind="attend", B=1, new=1, ctx=1023, H=12, Hkv=12, D=64, page=64, name="attend_one"),
        # 32 sequences generate together near the full 8192-token context: the cache's bytes
        dict(kind="attend", B=32, new=1, ctx=8191, H=16, Hkv=16, D=128, page=64,
             name="attend_generate"),
        # long prompts enter in chunks of 2048 tokens: matrix-core bound
        dict(kind="attend", B=4, new=2048, ctx=14336, H=16, Hkv=16, D=128, page=64,
             even=True, name="attend_prompt"),
        # generation with shared heads, weights kept for a later eviction
        dict(kind="track", B=8, new=1, ctx=8191, H=32, Hkv=8, D=128, page=32, name="track_generate"),
        # a ragged batch of prompt pieces and single tokens, shared heads, small pages
        dict(kind="track", B=7, new=301, ctx=3001, H=16, Hkv=4, D=64, page=16, name="track_ragged"),
        # one sequence at its budget's end
        dict(kind="evict", B=1, new=0, ctx=1100, H=12, Hkv=12, D=64, page=64, budget=1000,
             recent=64, name="evict_one"),
        # a batch of long sequences halved
        dict(kind="evict", B=16, new=0, ctx=8192, H=16, Hkv=16, D=128, page=64, budget=4096,
             recent=256, name="evict_batch"),
        # the next token of 16 sequences that generate together, 50,432-token vocabulary
        dict(kind="logprob", rows=16, V=50432, top=8, wide=False, f32=False, name="logprob_generate"),
        # texts scored under a vocabulary that no vector length divides, fp32 logits
        dict(kind="logprob", rows=1501, V=50277, top=5, wide=False, f32=True, name="logprob_score"),
        # loss of a 16,384-token quarter of a training step, with its gradient
        dict(kind="loss", rows=16384, V=50432, top=0, wide=False, f32=False, name="loss_step"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["append", "attend", "attend", "attend", "track", "track", "evict", "logprob",
                       "logprob", "loss"])
    if kind in ("logprob", "loss"):
        V = _log_int(rng, 64, 131072)
        if rng.random() < 0.5:  # a vocabulary padded for the products; the others are of any size
            V = max(64, V // 64 * 64)
        rows = min(_log_int(rng, 1, 16384), 16384 * 50432 // V)
        if kind == "logprob":  # (the plain form holds a whole number of 64 bits for each logit)
            rows = max(1, min(rows, 2048 * 50432 // V))
        return dict(kind=kind, rows=rows, V=V, top=rng.randint(1, 20) if kind == "logprob" else 0,
                    wide=rng.random() < 0.3, f32=rng.random() < 0.4)
    H, Hkv, D = rng.choice([(12, 12, 64), (16, 16, 64), (16, 16, 128), (32, 32, 128), (16, 4, 64),
                            (32, 8, 128), (12, 4, 128), (16, 1, 64), (14, 2, 128)])
    case = dict(kind=kind, B=_log_int(rng, 1, 32), new=0, ctx=_log_int(rng, 16, 14336), H=H, Hkv=Hkv,
                D=D, page=rng.choice([16, 32, 64, 128]))
    if kind == "evict":
        case["ctx"] = max(64, case["ctx"])
        # no more rows than the listed ones hold
        case["B"] = max(1, min(case["B"], 16 * 8192 * 16 * 128 // (case["ctx"] * Hkv * D)))
        case["budget"] = rng.randint(case["ctx"] // 8, case["ctx"])
        case["recent"] = rng.randint(0, case["budget"] // 2)
        return case
    case["new"] = 1 if rng.random() < 0.4 else _log_int(rng, 1, 2048)
    # bounds of the listed cases: cached elements, scores of the plain form
    per = (case["ctx"] + case["new"]) * Hkv * D
    case["B"] = max(1, min(case["B"], 32 * 8192 * 16 * 128 // per,
                           3 * 16 * 2048 * 16384 // (H * case["new"] * (case["ctx"] + case["new"]))))
    return case


def _lengths(case):
    """(slots in use, new tokens) of each sequence: an even batch, or a ragged
    one of which the first sequence has the most of both; where tokens come in
    chunks, one sequence of three or more has none and one begins."""
    rng = random.Random(case["B"] * 7919 + case["ctx"] * 31 + case["new"])
    B, ctx, new = case["B"], case["ctx"], case["new"]
    if case.get("even"):
        return [ctx] * B, [new] * B
    lens = [ctx] + [rng.randint(ctx // 2, ctx) for _ in range(B - 1)]
    news = [new] + [rng.choice([new, rng.randint(1, max(1, new))]) for _ in range(B - 1)]
    if new > 1 and B > 2:
        news[1], lens[2] = 0, 0  # nothing to do; the first chunk of a sequence
    if case["kind"] == "evict":
        news = [0] * B
    return lens, news


# ---------------------------------------------------------------------------
# inputs


def _bf16(x):
    return x.to(torch.bfloat16)


def _normal(gen, *shape):
    return torch.randn(shape, generator=gen, device=DEVICE, dtype=torch.float32)


def _uniform(gen, *shape):
    return torch.rand(shape, generator=gen, device=DEVICE, dtype=torch.float32)


def _ints(values):
    return torch.tensor(values, dtype=torch.int32, device=DEVICE)


def _logit_inputs(case, gen):
    """Logits of a trained model: a background, some tokens that stand out,
    the given token among them more often than not; upstream gradients of a
    mean over the tokens."""
    rows, V = case["rows"], case["V"]
    wide = V + 56 if case["wide"] else V
    x = torch.empty((rows, wide), dtype=torch.float32 if case["f32"] else torch.bfloat16,
                    device=DEVICE)
    for at in range(0, rows, 4096):
        n = min(4096, rows - at)
        x[at:at + n] = 2.5 * _normal(gen, n, wide) + 3 * _normal(gen, 1, wide)
    x = x[:, :V]
    targets = (_uniform(gen, rows) * V).long().clamp_(max=V - 1)
    likely = torch.randint(0, V, (rows, 8), generator=gen, device=DEVICE)
    at = torch.arange(rows, device=DEVICE)[:, None]
    x[at, likely] += (8 * _uniform(gen, rows, 8)).to(x.dtype)
    targets = torch.where(_uniform(gen, rows) < 0.6, likely[:, 0], targets)
    t = {"logits": x, "targets": targets}
    if case["kind"] == "loss":
        t["g_logp"] = -(0.5 + _uniform(gen, rows)) / rows
        t["g_entropy"] = 0.01 * _normal(gen, rows) / rows
        t["g_lse"] = 2e-4 * (8 + 4 * _normal(gen, rows)) / rows
    return t


def _inputs(case, seed):
    """The tensors of a pass, by name, from the seed alone."""
    gen = torch.Generator(device=DEVICE).manual_seed(int(seed))
    kind = case["kind"]
    if kind in ("logprob", "loss"):
        return _logit_inputs(case, gen)
    B, H, Hkv, D, page = (case[n] for n in ("B", "H", "Hkv", "D", "page"))
    lens, news = _lengths(case)
    per = max(-(-(a + n) // page) for a, n in zip(lens, news))
    pages = B * per
    t = {"lens": _ints(lens), "page": page,
         "table": torch.randperm(pages, generator=gen, device=DEVICE).int().view(B, per)}
    k, v = (torch.empty((pages, Hkv, page, D), dtype=torch.bfloat16, device=DEVICE)
            for _ in range(2))
    for at in range(0, pages, 4096):
        n = min(4096, pages - at)
        # keys: channels of different size, as after training
        k[at:at + n] = _normal(gen, n, Hkv, page, D) * torch.exp(0.3 * _normal(gen, D))
        v[at:at + n] = _normal(gen, n, Hkv, page, D) + 0.5 * _normal(gen, 1, Hkv, 1, D)
    t["k_pages"], t["v_pages"] = k, v
    slots = per * page
    if kind == "evict":
        t["weights"] = torch.exp(2 * _normal(gen, B, Hkv, slots) - 1)
        gaps = (1 + 2 * _uniform(gen, B, Hkv, slots)).int()
        t["positions"] = torch.cumsum(gaps, dim=2, dtype=torch.int32)
        last = torch.gather(t["positions"], 2, (t["lens"].long() - 1)[:, None, None].expand(B, Hkv, 1))
        t["seen"] = last.amax(dim=(1, 2)).int() + 1
        t["budget"], t["recent"] = case["budget"], case["recent"]
        return t
    cu = [0]
    for n in news:
        cu.append(cu[-1] + n)
    t["cu_new"] = _ints(cu)
    t["new"] = max(news)
    t["q"] = _bf16(1.2 * _normal(gen, cu[-1], H, D))
    if kind == "append":
        # the columns of one projection's output
        kv = _bf16(_normal(gen, cu[-1], 2, Hkv, D))
        t["k"], t["v"] = kv[:, 0], kv[:, 1]
        # positions run ahead of the slots where some were evicted
        t["start"] = t["lens"] + (200 * _uniform(gen, B)).int()
        t["positions"] = torch.zeros((B, Hkv, slots), dtype=torch.int32, device=DEVICE)
    if kind == "track":
        t["weights"] = torch.exp(2 * _normal(gen, B, Hkv, slots) - 1)
        t["weights_out"] = torch.zeros_like(t["weights"])
    return t


def prepare(case, seed):
    return {"kind": case["kind"], "top": case.get("top", 0), "t": _inputs(case, seed)}


# ---------------------------------------------------------------------------
# one pass


def run(state):
    kind, t = state["kind"], state["t"]
    if own:
        return _run_own(kind, t, state["top"])
    if kind == "append":
        return _append(t)
    if kind in ("attend", "track"):
        return _attend(t, kind == "track")
    if kind == "evict":
        return _evict(t)
    return _logits(t, state["top"], kind == "loss")


def _run_own(kind, t, top):
    import paper_2405_13226_amd as dd
    if kind == "append":
        q = dd.cache_append(t["q"], t["k"], t["v"], t["k_pages"], t["v_pages"], t["table"],
                            t["lens"], t["cu_new"], rope_base=ROPE_BASE, start=t["start"],
                            positions=t["positions"])
        return q, t["k_pages"], t["v_pages"], t["positions"]
    if kind == "attend":
        return dd.cache_attention(t["q"], t["k_pages"], t["v_pages"], t["table"], t["lens"],
                                  t["cu_new"])
    if kind == "track":
        o, lse = dd.cache_attention(t["q"], t["k_pages"], t["v_pages"], t["table"], t["lens"],
                                    t["cu_new"], weights=t["weights"],
                                    weights_out=t["weights_out"])
        return o, lse, t["weights_out"]
    if kind == "evict":
        weights, positions, lens = dd.cache_evict(t["k_pages"], t["v_pages"], t["table"], t["lens"],
                                                  t["weights"], t["positions"], t["seen"],
                                                  t["budget"], t["recent"])
        n = t["budget"]  # the slots that are defined; what lies behind them is no output
        return t["k_pages"], t["v_pages"], weights[..., :n], positions[..., :n], lens
    if kind == "logprob":
        return dd.logprobs(t["logits"], t["targets"], top=top)
    logp, entropy, lse = dd.logprobs(t["logits"], t["targets"])
    grad = dd.logprobs_backward(t["logits"], t["targets"], lse, entropy, t["g_logp"],
                                t["g_entropy"], t["g_lse"])
    return logp, entropy, lse, grad


def _rows(t):
    """(sequence, place in its chunk) of each row of the chunk."""
    cu = t["cu_new"].long()
    n = t["q"].shape[0]
    row = torch.arange(n, device=DEVICE)
    b = torch.searchsorted(cu, row, right=True) - 1
    return b, row - cu[b]


def _append(t):
    b, i = _rows(t)
    q, k, v, page = t["q"], t["k"], t["v"], t["page"]
    D = q.shape[2]
    pos = t["start"][b].long() + i
    freq = ROPE_BASE ** (-torch.arange(0, D, 2, device=DEVICE, dtype=torch.float64) / D)
    angle = pos[:, None].double() * freq
    angle = torch.remainder(angle, 2 * math.pi)
    c, s = torch.cos(angle).float()[:, None], torch.sin(angle).float()[:, None]

    def rotated(x):
        a, z = x[..., 0::2].float(), x[..., 1::2].float()
        return _bf16(torch.stack([a * c - z * s, a * s + z * c], dim=-1).flatten(-2))

    slot = t["lens"][b].long() + i
    p, at = t["table"][b, slot // page].long(), slot % page
    t["k_pages"][p, :, at] = rotated(k)
    t["v_pages"][p, :, at] = v
    t["positions"][b, :, slot] = pos.int()[:, None]
    return rotated(q), t["k_pages"], t["v_pages"], t["positions"]


def _gather(pages, table):
    """[B, kv heads, slots, D] in fp32 of the sequences' pages."""
    x = pages[table.long()].float()
    return x.transpose(1, 2).flatten(2, 3)


def _attend(t, track):
    q, lens = t["q"], t["lens"].long()
    T, H, D = q.shape
    B, n = t["table"].shape[0], t["new"]
    Hkv = t["k_pages"].shape[1]
    G = H // Hkv
    b, i = _rows(t)
    padded = torch.zeros((B, n, H, D), device=DEVICE)
    padded[b, i] = q.float()
    # rows of a key head: the chunk's tokens, and the heads that share it
    rows = padded.view(B, n, Hkv, G, D).transpose(1, 2).reshape(B, Hkv, n * G, D)
    k, v = _gather(t["k_pages"], t["table"]), _gather(t["v_pages"], t["table"])
    s = torch.matmul(rows, k.transpose(2, 3)) * (1 / math.sqrt(D))
    slot = torch.arange(k.shape[2], device=DEVICE)
    token = torch.arange(n * G, device=DEVICE) // G
    hidden = slot > (lens[:, None] + token)[:, None, :, None]
    s.masked_fill_(hidden, -math.inf)
    top = s.amax(dim=-1, keepdim=True)
    p = torch.exp_(s.sub_(top))
    total = p.sum(dim=-1, keepdim=True)
    lse = (top + torch.log(total)).view(B, Hkv, n, G).transpose(1, 2).reshape(B, n, H)[b, i]
    p.div_(total)
    # slots behind a sequence's last hold what others left
    live = slot < (lens + (t["cu_new"][1:] - t["cu_new"][:-1]))[:, None]
    v.masked_fill_(~live[:, None, :, None], 0)
    o = torch.matmul(p, v).view(B, Hkv, n, G, D).transpose(1, 2).reshape(B, n, H, D)[b, i]
    if not track:
        return _bf16(o), lse
    new = token < (t["cu_new"][1:] - t["cu_new"][:-1])[:, None]
    w = (p * new[:, None, :, None]).sum(dim=2)
    w += torch.where(slot < lens[:, None], 1.0, 0.0)[:, None] * t["weights"]
    t["weights_out"].copy_(torch.where(live[:, None], w, t["weights_out"]))
    return _bf16(o), lse, t["weights_out"]


def _evict(t):
    w, pos, lens, budget, page = (t[n] for n in ("weights", "positions", "lens", "budget", "page"))
    B, Hkv, slots = w.shape
    slot = torch.arange(slots, device=DEVICE)
    live = (slot < lens[:, None, None]).expand(B, Hkv, slots)
    protected = live & (pos >= (t["seen"] - t["recent"])[:, None, None])
    rank = torch.where(live, w, -math.inf)
    rank = torch.where(protected, math.inf, rank)
    order = torch.sort(rank, dim=-1, descending=True, stable=True).indices
    kept = torch.zeros_like(live).scatter_(2, order[..., :budget], True)
    full = (lens > budget)[:, None, None]
    kept &= live
    holes, extra = full & ~kept & (slot < budget), full & kept & (slot >= budget)
    # the n-th hole takes the n-th survivor behind the budget
    bh, hh, to = torch.nonzero(holes, as_tuple=True)
    be, he, src = torch.nonzero(extra, as_tuple=True)
    new_w, new_pos = w.clone(), pos.clone()
    new_w[bh, hh, to], new_pos[bh, hh, to] = w[be, he, src], pos[be, he, src]
    table = t["table"].long()
    for pages in (t["k_pages"], t["v_pages"]):
        pages[table[bh, to // page], hh, to % page] = pages[table[be, src // page], he, src % page]
    return (t["k_pages"], t["v_pages"], new_w[..., :budget], new_pos[..., :budget],
            torch.clamp(lens, max=budget))


def _logits(t, top, gradient):
    x, targets = t["logits"].float(), t["targets"]
    best = x.amax(dim=-1, keepdim=True)
    p = torch.exp(x - best)
    total = p.sum(dim=-1, keepdim=True)
    p.div_(total)
    lse = best + torch.log(total)
    given = torch.gather(x, 1, targets[:, None])
    entropy = torch.log(total) - (p * (x - best)).sum(dim=-1, keepdim=True)
    out = (given - lse)[:, 0], entropy[:, 0], lse[:, 0]
    if gradient:
        g_logp, g_h, g_lse = (t[n][:, None] for n in ("g_logp", "g_entropy", "g_lse"))
        d = p * (g_lse - g_logp - g_h * (x - lse + entropy))
        d.scatter_add_(1, targets[:, None], g_logp)
        return (*out, d.to(t["logits"].dtype))
    if top:
        # values in order as whole numbers, equal ones by the lowest index
        u = x.contiguous().view(torch.int32).long()
        u = torch.where(u < 0, -(u & 0x7fffffff), u)
        V = x.shape[1]
        key = torch.topk(u * V + torch.arange(V - 1, -1, -1, device=DEVICE), top, dim=-1).values
        ids = V - 1 - torch.remainder(key, V)
        return (*out, torch.gather(x, 1, ids) - lse, ids)
    return out


# ---------------------------------------------------------------------------
# what a pass cannot do without


def work(case):
    kind = case["kind"]
    if kind in ("logprob", "loss"):
        rows, V, size = case["rows"], case["V"], 4 if case["f32"] else 2
        if kind == "logprob":
            return {"bytes": rows * (V * size + 8 + 12 + 12 * case["top"]), "flops": 6 * rows * V}
        return {"bytes": rows * (2 * V * size + 8 + 24), "flops": 12 * rows * V}
    H, Hkv, D = case["H"], case["Hkv"], case["D"]
    lens, news = _lengths(case)
    T = sum(news)
    if kind == "append":
        return {"bytes": T * ((2 * H + 4 * Hkv) * D * 2 + 4 * Hkv), "flops": T * (H + Hkv) * D * 3}
    if kind == "evict":
        n = case["budget"]
        moved = sum(n * (a - n) / a for a in lens if a > n)
        return {"bytes": int(Hkv * (8 * sum(lens) + 8 * sum(min(a, n) for a in lens)
                                    + moved * 8 * D)), "flops": 0}
    used = sum(a + n for a, n in zip(lens, news) if n)
    pairs = sum(n * a + n * (n + 1) // 2 for a, n in zip(lens, news))
    size = 2 * T * H * D * 2 + 4 * T * H + 2 * used * Hkv * D * 2
    if kind == "track":
        size += 8 * used * Hkv
    return {"bytes": size, "flops": 4 * D * H * pairs}


# ---------------------------------------------------------------------------
# the same outputs from the definition in 64 bits


def exact(case, seed):
    t = _inputs(case, seed)
    kind = case["kind"]
    if kind in ("logprob", "loss"):
        return _exact_logits(t, case["top"], kind == "loss")
    if kind == "evict":
        return None  # nothing is computed: rows move as they are
    lens, news = _lengths(case)
    return _exact_append(t, lens, news) if kind == "append" else _exact_attend(t, lens, news)


def _exact_append(t, lens, news):
    D, page = t["q"].shape[2], t["page"]
    start = t["start"].tolist()
    pos = torch.cat([a + torch.arange(n, dtype=torch.float64) for a, n in zip(start, news)])
    turn = torch.exp(torch.arange(D // 2, dtype=torch.float64) * (-2 / D * math.log(ROPE_BASE)))
    angle = (pos[:, None, None] * turn).to(DEVICE)
    unit = torch.polar(torch.ones_like(angle), angle)

    def rotated(x):
        z = torch.view_as_complex(x.double().reshape(*x.shape[:2], D // 2, 2))
        return torch.view_as_real(z * unit).reshape(x.shape)

    q, k = rotated(t["q"]), rotated(t["k"])
    pages, first = t["k_pages"].double(), 0
    for b, (used, n) in enumerate(zip(lens, news)):
        slot = torch.arange(used, used + n, device=DEVICE)
        pages[t["table"][b].long()[slot // page], :, slot % page] = k[first:first + n]
        first += n
    return q, pages, None, None


def _exact_attend(t, lens, news):
    q, page = t["q"], t["page"]
    T, H, D = q.shape
    Hkv = t["k_pages"].shape[1]
    G = H // Hkv
    o = torch.zeros((T, H, D), dtype=torch.float64, device=DEVICE)
    lse = torch.zeros((T, H), dtype=torch.float64, device=DEVICE)
    w = t["weights_out"].double() if "weights" in t else None
    first = 0
    for b, (used, n) in enumerate(zip(lens, news)):
        total = used + n
        ids = t["table"][b, :-(-total // page)].long() if total else None
        for h in range(Hkv) if total else ():
            k, v = (t[p][ids, h].reshape(-1, D)[:total].double() for p in ("k_pages", "v_pages"))
            if w is not None:
                w[b, h, :used] = t["weights"][b, h, :used].double()
                w[b, h, used:total] = 0
            for at in range(0, n, 512):
                m = min(512, n - at)
                rows = slice(first + at, first + at + m)
                x = q[rows, h * G:(h + 1) * G].double()
                s = torch.tensordot(x, k, dims=([2], [1])) * D ** -0.5
                seen = torch.arange(total, device=DEVICE)[None] <= \
                    used + at + torch.arange(m, device=DEVICE)[:, None]
                s = torch.where(seen[:, None], s, -math.inf)
                z = torch.logsumexp(s, dim=2)
                p = torch.exp(s - z[:, :, None])
                o[rows, h * G:(h + 1) * G] = torch.tensordot(p, v, dims=1)
                lse[rows, h * G:(h + 1) * G] = z
                if w is not None:
                    w[b, h, :total] += p.sum(dim=(0, 1))
        first += n
    return (o, lse) if w is None else (o, lse, w)


def _exact_logits(t, top, gradient):
    x, targets = t["logits"], t["targets"]
    parts = []
    for at in range(0, x.shape[0], 2048):
        rows = slice(at, at + 2048)
        y = x[rows].double()
        lp = torch.log_softmax(y, dim=1)
        z = torch.logsumexp(y, dim=1)
        p = lp.exp()
        h = -(p * lp).sum(dim=1)
        part = [lp[torch.arange(len(y), device=DEVICE), targets[rows]], h, z]
        if gradient:
            g = [t[n][rows].double()[:, None] for n in ("g_logp", "g_entropy", "g_lse")]
            d = -g[0] * p - g[1] * p * (lp + h[:, None]) + g[2] * p
            d[torch.arange(len(y), device=DEVICE), targets[rows]] += g[0][:, 0]
            part.append(d)
        elif top:
            part.append(torch.topk(lp, top, dim=1).values)
        parts.append(part)
    out = [torch.cat(c) for c in zip(*parts)]
    return (*out, None) if top and not gradient else tuple(out)

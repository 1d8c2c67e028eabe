"""The paged cache's operators and the log probabilities in float64, from their
definitions (CPU tensors; nothing of the package is used), and ragged batches
to try them on."""
import math

import torch

U = 2.0 ** -24   # half a step of fp32, relative
HB = 2.0 ** -8   # of bf16


class Batch:
    """A cache of random contents in shuffled pages with a ragged chunk:
    lens[b] slots in use, news[b] new tokens.  Table entries behind the pages in
    use name no page."""

    def __init__(self, lens, news, H, Hkv, D, page, seed=0, spare=1, tail=0, scale=1.0):
        g = torch.Generator().manual_seed(seed)
        self.lens, self.news, self.page = list(lens), list(news), page
        self.H, self.Hkv, self.D, self.B = H, Hkv, D, len(lens)
        used = [-(-(a + n) // page) for a, n in zip(lens, news)]
        self.per = max(max(used), 1) + spare
        self.pages = max(sum(used), 1) + 2
        order = torch.randperm(self.pages, generator=g).tolist()
        rows = []
        for u in used:
            ids = [order.pop() for _ in range(u)]
            rows.append(ids + [(-1, 2 ** 31 - 1, -2 ** 31)[i % 3] for i in range(self.per - u)])
        self.table = torch.tensor(rows, dtype=torch.int32)
        self.T = sum(news) + tail
        cu = [0]
        for n in news:
            cu.append(cu[-1] + n)
        self.cu = torch.tensor(cu, dtype=torch.int32)
        self.lens_t = torch.tensor(self.lens, dtype=torch.int32)
        self.slots = self.per * page

        def normal(*shape):
            return torch.randn(*shape, generator=g)
        shape = (self.pages, Hkv, page, D)
        self.k, self.v = (normal(*shape).to(torch.bfloat16) for _ in range(2))
        self.q = (scale * normal(self.T, H, D)).to(torch.bfloat16)
        self.w = torch.rand(self.B, Hkv, self.slots, generator=g)
        self.g = g

    def slot_rows(self, pages, b, h, n):
        """Slots 0 .. n - 1 of head h of sequence b."""
        ids = self.table[b, :-(-n // self.page)].long()
        return pages[ids, h].reshape(-1, self.D)[:n]

    def to(self, dev):
        return {n: getattr(self, n).to(dev) for n in ("table", "cu", "lens_t", "k", "v", "q", "w")}


def attention(x):
    """(o, lse, weights) and the elementwise tolerances of each for the batch x:

    * a score is a sum of D products, at most D + 2 fp32 roundings of the
      magnitudes added, and its exponent's argument three of its own size (the
      running maximum's among them): `e` in the exponent, so 2 e of a
      probability (numerator and denominator);
    * the row's sum and the join of its parts: n + 80 roundings; exponentials
      and reciprocals a few each: (n + 100) u of everything;
    * probabilities are rounded to bf16 for their product with V, o once more.
    """
    o = torch.zeros(x.T, x.H, x.D, dtype=torch.float64)
    lse = torch.zeros(x.T, x.H, dtype=torch.float64)
    to, tl = torch.zeros_like(o), torch.zeros_like(lse)
    w, tw = x.w.double().clone(), torch.zeros(x.w.shape, dtype=torch.float64)
    G = x.H // x.Hkv
    first = 0
    for b, (used, n) in enumerate(zip(x.lens, x.news)):
        total = used + n
        for h in range(x.Hkv if total else 0):
            k, v = (x.slot_rows(p, b, h, total).double() for p in (x.k, x.v))
            add, ta = torch.zeros(total, dtype=torch.float64), torch.zeros(total, dtype=torch.float64)
            for i in range(n):
                m = used + i + 1
                q = x.q[first + i, h * G:(h + 1) * G].double()
                s = (q @ k[:m].T) / math.sqrt(x.D)
                z = torch.logsumexp(s, dim=1)
                p = torch.exp(s - z[:, None])
                size = (q.abs() @ k[:m].abs().T) / math.sqrt(x.D)
                e = ((x.D + 2) * U * size + 3 * U * (s.abs() + z.abs()[:, None] + 16)).amax(dim=1)
                rel = 2 * e + (m + 100) * U
                rows = slice(h * G, (h + 1) * G)
                o[first + i, rows] = p @ v[:m]
                to[first + i, rows] = HB * (p @ v[:m]).abs() + \
                    (HB + rel[:, None]) * (p @ v[:m].abs()) * 1.01
                lse[first + i, rows] = z
                tl[first + i, rows] = e + (m + 100) * U + 4 * U * z.abs()
                add[:m] += p.sum(dim=0)
                ta[:m] += (p * rel[:, None]).sum(dim=0) + (n * G + 8) * U * p.sum(dim=0)
            base = x.w[b, h, :total].double()
            base[used:] = 0
            w[b, h, :total] = base + add
            tw[b, h, :total] = ta + 2 * U * (base + add)
        first += n
    return (o, lse, w), (to, tl, tw)


def rotate(q, pos, base):
    """q [T, heads, D] rotated at positions pos, in float64."""
    D = q.shape[-1]
    freq = torch.exp(torch.arange(D // 2, dtype=torch.float64) * (-2 / D * math.log(base)))
    a = pos.double()[:, None, None] * freq
    x0, x1 = q.double()[..., 0::2], q.double()[..., 1::2]
    return torch.stack([x0 * a.cos() - x1 * a.sin(), x0 * a.sin() + x1 * a.cos()], -1).flatten(-2)


def evict(lens, w, pos, seen, budget, recent):
    """For each (sequence, head): (slot that receives, slot it comes from) in
    order, in plain Python."""
    B, Hkv, _ = w.shape
    moves = {}
    for b in range(B):
        n = int(lens[b])
        for h in range(Hkv):
            if n <= budget:
                moves[b, h] = []
                continue

            def rank(j):
                x = float(w[b, h, j])
                if int(pos[b, h, j]) >= int(seen[b]) - recent:
                    return (0, 0.0, j)
                return (2, 0.0, j) if math.isnan(x) else (1, -x, j)
            kept = sorted(sorted(range(n), key=rank)[:budget])
            holes = sorted(set(range(budget)) - set(kept))
            moves[b, h] = list(zip(holes, [j for j in kept if j >= budget]))
    return moves


def logprobs(x, targets, top=0):
    """(logp, entropy, lse[, top_logp, ids]) in float64."""
    x = x.double()
    best = x.amax(dim=1, keepdim=True)
    e = torch.exp(x - best)
    total = torch.log(e.sum(dim=1))
    z = best[:, 0] + total
    # (not x - z: rows near fp32's lowest number leave nothing of the sum in z)
    lp = (x - best) - total[:, None]
    p = torch.exp(lp)
    h = -torch.where(p > 0, p * lp, 0.0).sum(dim=1)
    given = torch.gather(lp, 1, targets.clamp(min=0)[:, None])[:, 0]
    out = [torch.where(targets < 0, 0.0, given), h, z]
    if top:
        ids = torch.sort(x, dim=1, descending=True, stable=True).indices[:, :top]
        out += [torch.gather(lp, 1, ids), ids]
    return out


def logprobs_grad(x, targets, g_logp, g_entropy, g_lse):
    """(gradient, sum of the magnitudes that it is formed from) in float64."""
    _, h, z = logprobs(x, targets)[:3]
    lp = x.double() - z[:, None]
    p = torch.exp(lp)
    lp = torch.where(p > 0, lp, 0.0)
    gl = torch.where(targets < 0, 0.0, g_logp.double())[:, None]
    ge, gz = g_entropy.double()[:, None], g_lse.double()[:, None]
    one = torch.zeros_like(p)
    one.scatter_(1, targets.clamp(min=0)[:, None], 1.0)
    d = gl * (one - p) + gz * p - ge * p * (lp + h[:, None])
    size = gl.abs() * (one + p) + gz.abs() * p + ge.abs() * p * (lp.abs() + h[:, None])
    return d, size

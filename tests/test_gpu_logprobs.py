"""GPU parity of the log probabilities and their gradient against float64.

Tolerances, elementwise, u = 2^-24 (the fp32 rounding, relative):

* lse: e^(x - m) has the exponent's rounding (2 u of |x - m| <= `far`, the
  row's largest useful distance, 100 here: what lies further adds less than
  e^-100) and the exponential's; a thread's sums, the wave's and the workgroup's
  tree and the parts are below V / 256 + 100 additions: `r` = (2 far + V / 256 +
  110) u relative, so r absolute in the logarithm, and 4 u of |m| + |log|.
* logp: twice that (one more subtraction).  entropy: H = log s - u / s, each
  with r of its size; the size of u / s is at most `far` + log V.
* gradient: p has 2 (the lse's tolerance) + 4 u (|x - lse| + 1) relative; the
  rest are a few roundings of the magnitudes added, and one to the logits' type.
"""
import math

import pytest
import torch

import paper_2405_13226_amd as dd

import cache_oracle as O
from cache_oracle import HB, U
from parity import log

pytestmark = pytest.mark.gpu

# rows, V, top: one logit; less than a piece, a wave, a workgroup; sizes that
# nothing divides; rows split over workgroups and not
SHAPES = [(1, 1, 1), (3, 2, 2), (5, 7, 3), (4, 64, 64), (33, 65, 0), (2, 511, 5), (7, 513, 20),
          (1, 2049, 8), (600, 1000, 4), (1, 4096, 1), (3, 12345, 64), (16, 50432, 8), (2, 50277, 20),
          (1, 131072, 33), (700, 9001, 3),
          (1100, 2200, 6), (1100, 2201, 6)]


def tolerances(x, ref):
    V = x.shape[1]
    z = ref[2].abs()
    r = (200 + V / 256 + 110) * U
    t_lse = r + 4 * U * (z + 20)
    t_h = r * (100 + math.log(V)) / 10 + 4 * U * (ref[1].abs() + 20)
    return 2 * t_lse, t_h, t_lse


def close(got, ref, tol, what):
    got = got.double().cpu()
    assert got.shape == ref.shape, what
    # (infinite where the value is, or leaves fp32's range)
    far = torch.isinf(ref.float())
    same = torch.equal(got[far], ref[far].float().double())
    assert same and bool(torch.isfinite(got[~far]).all()), what
    off = ((got - ref).abs() - tol)[~far]
    assert bool((off <= 0).all()), (what, float(off.max()))


def case(rows, V, dtype, seed, scale=3.0):
    g = torch.Generator().manual_seed(seed)
    x = (scale * torch.randn(rows, V, generator=g) + torch.randn(1, V, generator=g)).to(dtype)
    t = torch.randint(0, V, (rows,), generator=g)
    t[torch.rand(rows, generator=g) < 0.2] = -100
    return x, t, [torch.randn(rows, generator=g) for _ in range(3)]


def check_forward(x, t, top, dev, xg=None):
    xg = x.to(dev) if xg is None else xg
    got = dd.logprobs(xg, t.to(dev), top=top)
    ref = O.logprobs(x, t, top)
    tl, th, tz = tolerances(x, ref)
    close(got[0], ref[0], tl * (t >= 0), "logp")
    close(got[1], ref[1], th, "entropy")
    close(got[2], ref[2], tz, "lse")
    if top:
        assert torch.equal(got[4].cpu(), ref[4])
        close(got[3], ref[3], tl[:, None] + 2 * U * ref[3].abs(), "top")
        plain = dd.logprobs(xg, t.to(dev))
        # (the split differs where alternatives are few)
        close(plain[2], ref[2], tz, "lse without alternatives")
    return got


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("rows,V,top", SHAPES)
def test_forward(cuda, rows, V, top, dtype):
    log(f"logprobs {rows} x {V} top {top} {dtype}")
    x, t, _ = case(rows, V, dtype, rows + V)
    check_forward(x, t, top, cuda)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_ties_order_and_extremes(cuda, dtype):
    log(f"logprobs: ties, order, extremes {dtype}")
    V = 6000
    rows = [torch.zeros(V), torch.arange(V).float() / 64, -torch.arange(V).float() / 64,
            torch.randint(0, 3, (V,)).float(), torch.full((V,), torch.finfo(dtype).min),
            torch.full((V,), 80.0), torch.where(torch.arange(V) % 2 == 0, 0.0, -0.0)]
    a = torch.randn(V)
    a[100:] = float("-inf")  # fewer finite ones than a wave's piece
    b = torch.full((V,), float("-inf"))
    b[77] = 5.0
    c = torch.full((V,), torch.finfo(dtype).min)
    c[5990] = torch.finfo(dtype).max
    x = torch.stack(rows + [a, b, c]).to(dtype)
    t = torch.tensor([3, 5, 0, 7, 9, 11, 1, 50, 77, 5990])
    check_forward(x, t, 40, cuda)


# a wave, a workgroup of 256 and of 1024, several of them per row
@pytest.mark.parametrize("rows,V", [(5, 2000), (5, 8000), (5, 30000), (5, 150000), (600, 20000),
                                    (2100, 4200)])
def test_equal_logits_and_neighbours(cuda, rows, V):
    """Lists of alternatives that do not fit (all logits equal, or two values),
    alternatives that lie next to each other, and ones of one thread's pieces."""
    log(f"logprobs: equal logits {rows} x {V}")
    x = torch.zeros(rows, V)
    x[1] = torch.arange(V) % 2
    x[2:4] = torch.randn(2, V).clamp(max=3)
    x[2, V // 2:V // 2 + 30] = 8 + torch.arange(30) % 7
    for step in (64 * 8, 256 * 8, 1024 * 8):
        x[3, 8:8 + step * 12:step][:12] = 9.0
    x[4:] = torch.randn(rows - 4, 1)
    for dtype in (torch.bfloat16, torch.float32):
        y = x.to(dtype)
        for top in (1, 20, 64):
            check_forward(y[:5], torch.zeros(5, dtype=torch.int64), top, cuda)
        ids = dd.logprobs(y.to(cuda), torch.zeros(rows, dtype=torch.int64, device=cuda), top=9)[4]
        assert torch.equal(ids[:4].cpu(), O.logprobs(y[:4], torch.zeros(4).long(), 9)[4])
        assert (ids[4:] == torch.arange(9, device=cuda)).all()


def test_large_gradients_are_the_small_ones(cuda):
    """Past the size from which gradients are stored past the caches."""
    log("logprobs: gradients of more than 256 MB")
    for dtype, rows in ((torch.float32, 1400), (torch.bfloat16, 2800)):
        x = torch.randn(rows, 50277, device=cuda).to(dtype)
        t = torch.arange(rows, device=cuda)
        _, h, lse = dd.logprobs(x, t)
        g = torch.randn(3, rows, device=cuda)
        all_rows = dd.logprobs_backward(x, t, lse, h, *g)
        for part in (slice(0, rows // 2), slice(rows // 2, rows)):
            few = dd.logprobs_backward(x[part], t[part], lse[part], h[part], *(y[part] for y in g))
            assert torch.equal(all_rows[part], few)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("rows,V", [(2, 700), (2, 9000)])
def test_rows_out_of_the_ordinary(cuda, rows, V, dtype):
    """NaN and infinities stay in their rows; what is ignored or out of range."""
    log(f"logprobs: NaN, infinities, targets {dtype} {V}")
    x, _, g = case(6, V, dtype, 5)
    x[0, V // 2] = float("nan")
    x[1, V - 1] = float("inf")
    x[2] = float("-inf")
    t = torch.tensor([0, 0, 0, V, -1, 2])
    xd, td = x.to(cuda), t.to(cuda)
    logp, h, lse, best, ids = (y.cpu() for y in dd.logprobs(xd, td, top=V if V < 65 else 8))
    assert logp[:2].isnan().all() and h[:3].isnan().all() and lse[:2].isnan().all()
    assert lse[2] == float("-inf") and logp[2].isnan() and logp[3].isnan() and logp[4] == 0
    ref = O.logprobs(x[3:], torch.tensor([0, -1, 2]), 8)
    assert torch.equal(ids[3:], ref[4]) and torch.equal(ids[2], torch.arange(8))
    assert ids[1, 0] == V - 1 and not (ids[0] == V // 2).any()
    tl, th, tz = tolerances(x[3:], ref)
    close(lse[3:], ref[2], tz, "lse")
    close(h[3:], ref[1], th, "entropy")
    assert abs(float(logp[5]) - float(ref[0][2])) <= float(tl[2])
    # alternatives are fewer than asked for in no row, even of NaN alone
    y = torch.full((1, 50), float("nan"), dtype=dtype, device=cuda)
    ids = dd.logprobs(y, td[:1], top=50)[4]
    assert torch.equal(ids[0].cpu(), torch.arange(50))
    gd = [v.to(cuda) for v in g]
    dx = dd.logprobs_backward(xd, td, lse.to(cuda), h.to(cuda), *gd).cpu()
    assert dx[:2].isnan().all() and torch.isfinite(dx[4:]).all()


def check_backward(x, t, g, dev, xg=None, out=None):
    xg = x.to(dev) if xg is None else xg
    td, gd = t.to(dev), [y.to(dev) for y in g]
    _, h, lse = dd.logprobs(xg, td)
    dx = dd.logprobs_backward(xg, td, lse, h, *gd, out=out)
    ref, size = O.logprobs_grad(x, t, *g)
    r = O.logprobs(x, t)
    _, th, tz = tolerances(x, r)
    lp = (x.double() - r[2][:, None]).clamp(min=-200).abs()
    rel = 2 * tz[:, None] + 4 * U * (lp + 1) + 8 * U
    p = torch.exp(x.double() - r[2][:, None])
    tol = rel * size + p * (tz + th)[:, None] * g[1].double().abs()[:, None]
    tol = tol + (HB if x.dtype is torch.bfloat16 else U) * (ref.abs() + tol) + 1e-38
    close(dx, ref, tol, "gradient")
    return dx


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("rows,V", [(r, v) for r, v, _ in SHAPES])
def test_backward(cuda, rows, V, dtype):
    log(f"logprobs backward {rows} x {V} {dtype}")
    x, t, g = case(rows, V, dtype, rows + V)
    check_backward(x, t, g, cuda)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_masked_logits(cuda, dtype):
    """Logits of -inf and of the lowest finite value: no probability, gradient 0."""
    log(f"logprobs: masked logits {dtype}")
    x, t, g = case(8, 3001, dtype, 1)
    mask = torch.rand(8, 3001) < 0.5
    mask[torch.arange(8), t.clamp(min=0)] = False
    for value in (float("-inf"), torch.finfo(dtype).min):
        y = x.masked_fill(mask, value)
        check_forward(y, t, 7, cuda)
        dx = check_backward(y, t, g, cuda)
        assert (dx.cpu()[mask] == 0).all()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("rows,V", [(9, 1001), (3, 20000), (1, 333)])
def test_columns_of_a_wider_matrix(cuda, rows, V, dtype):
    """Any row stride and start; neighbours are neither read into a result nor
    written."""
    log(f"logprobs: columns {rows} x {V} {dtype}")
    x, t, g = case(rows, V, dtype, 2)
    wide = torch.full((rows, V + 13), float("nan"), dtype=dtype, device=cuda)
    for at in (1, 6):
        wide.fill_(float("nan"))
        part = wide[:, at:at + V]
        part.copy_(x)
        check_forward(x, t, 5, cuda, xg=part)
        out = torch.full((rows, V + 5), 7.0, dtype=dtype, device=cuda)
        check_backward(x, t, g, cuda, xg=part, out=out[:, 3:3 + V])
        assert (out[:, :3] == 7).all() and (out[:, 3 + V:] == 7).all()
        # in place
        ref = dd.logprobs_backward(x.to(cuda), t.to(cuda), *dd.logprobs(part, t.to(cuda))[2:0:-1],
                                   *[y.to(cuda) for y in g])
        _, h, lse = dd.logprobs(part, t.to(cuda))
        res = dd.logprobs_backward(part, t.to(cuda), lse, h, *[y.to(cuda) for y in g], out=part)
        assert res is part and torch.equal(part, ref)
        rest = torch.cat([wide[:, :at], wide[:, at + V:]], dim=1)
        assert rest.isnan().all()


def test_gradients_that_are_absent(cuda):
    log("logprobs: absent gradients")
    x, t, g = case(6, 500, torch.float32, 3)
    xd, td = x.to(cuda), t.to(cuda)
    _, h, lse = dd.logprobs(xd, td)
    zero = torch.zeros(6)
    for keep in range(8):
        some = [y if keep >> i & 1 else None for i, y in enumerate(g)]
        dx = dd.logprobs_backward(xd, td, lse, h, *[None if y is None else y.to(cuda) for y in some])
        full = dd.logprobs_backward(xd, td, lse, h, *[(zero if y is None else y).to(cuda)
                                                      for y in some])
        assert torch.equal(dx, full)


def test_autograd(cuda):
    """Through autograd, and against differences of the float64 definition."""
    log("logprobs: autograd")
    x, t, g = case(5, 40, torch.float32, 4)
    leaf = x.to(cuda).requires_grad_()
    logp, h, lse, best, ids = dd.token_logprobs(leaf, t.to(cuda), top=3)
    assert not best.requires_grad and not ids.requires_grad
    loss = (logp * g[0].to(cuda) + h * g[1].to(cuda)).sum() + 1e-2 * lse.square().sum()
    loss.backward()
    gz = 2e-2 * O.logprobs(x, t)[2]
    ref, _ = O.logprobs_grad(x, t, g[0], g[1], gz)
    assert ((leaf.grad.double().cpu() - ref).abs() <= 1e-5).all()

    def value(y):
        lp, hh, z = O.logprobs(y, t)
        return float((lp * g[0].double() + hh * g[1].double()).sum() + 1e-2 * (z * z).sum())
    for i, j in ((0, 0), (1, 7), (3, int(t[3].clamp(min=0))), (4, 39)):
        d = torch.zeros(5, 40, dtype=torch.float64)
        d[i, j] = 1e-5
        slope = (value(x.double() + d) - value(x.double() - d)) / 2e-5
        assert abs(slope - float(leaf.grad[i, j])) <= 1e-5 * (1 + abs(slope))
    # one result alone, and none
    leaf.grad = None
    dd.token_logprobs(leaf, t.to(cuda))[0].sum().backward()
    ref, _ = O.logprobs_grad(x, t, torch.ones(5), torch.zeros(5), torch.zeros(5))
    assert ((leaf.grad.double().cpu() - ref).abs() <= 1e-5).all()


def test_graph_and_streams(cuda):
    """A loss with its backward in a graph, replayed between eager work of the
    same leaf, and a call on another stream."""
    log("logprobs: graph")
    x, t, _ = case(40, 5000, torch.bfloat16, 6)
    td = t.to(cuda)
    xd = x.to(cuda)
    side = torch.cuda.Stream()

    def step():
        logp, h, lse, best, ids = dd.logprobs(xd, td, top=4)
        return logp, h, lse, best, ids, dd.logprobs_backward(xd, td, lse, h, g_logp=logp, g_lse=lse)
    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step()
    for i in range(3):
        xd.copy_(torch.randn_like(xd) * (i + 1))
        want = step()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, want))
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            other = step()
        torch.cuda.current_stream().wait_stream(side)
        assert all(torch.equal(a, b) for a, b in zip(other, want))


def test_rows_past_32_bits(cuda):
    log("logprobs: offsets past 32 bits")
    rows, V = 50000, 50432  # 2.5e9 logits
    x = torch.zeros(rows, V, dtype=torch.bfloat16, device=cuda)
    small, t, g = case(3, V, torch.bfloat16, 8)
    t = torch.tensor([1, 2, V - 1])
    x[-3:] = small.to(cuda)
    td = torch.zeros(rows, dtype=torch.int64, device=cuda)
    td[-3:] = t.to(cuda)
    logp, h, lse, best, ids = dd.logprobs(x, td, top=2)
    ref = O.logprobs(small, t, 2)
    tl, th, tz = tolerances(small, ref)
    close(logp[-3:], ref[0], tl, "logp")
    close(h[-3:], ref[1], th, "entropy")
    assert torch.equal(ids[-3:].cpu(), ref[4])
    assert (ids[:-3] == torch.tensor([0, 1], device=cuda)).all()
    gd = torch.ones(rows, device=cuda)
    gd[-3:] = g[0].to(cuda)
    dx = dd.logprobs_backward(x, td, lse, h, g_logp=gd, out=x)
    want, size = O.logprobs_grad(small, t, g[0], torch.zeros(3), torch.zeros(3))
    close(dx[-3:], want, HB * want.abs() + 1e-3 * size + 1e-30, "gradient")
    # rows of equal logits: 1 - 1/V at the target, -1/V elsewhere
    assert (dx[:-3, 1] == -torch.tensor(1 / V).to(torch.bfloat16).to(cuda)).all()


def test_empty(cuda):
    x = torch.zeros(0, 10, device=cuda)
    t = torch.zeros(0, dtype=torch.int64, device=cuda)
    out = dd.logprobs(x, t, top=2)
    assert [tuple(o.shape) for o in out] == [(0,), (0,), (0,), (0, 2), (0, 2)]
    z = torch.zeros(0, device=cuda)
    assert dd.logprobs_backward(x, t, z, z).shape == (0, 10)


def exact_grad(x, t, g_logp, g_entropy, g_lse):
    """(gradient, magnitudes, p, |log p|, entropy) in float64, log p = (x - m) -
    log sum e^(x - m): an lse in float64 does not hold that sum either where the
    logits are near fp32's largest."""
    a = x.double() - x.double().amax(dim=1, keepdim=True)
    lp = a - torch.log(torch.exp(a).sum(dim=1, keepdim=True))
    p = torch.exp(lp)
    lp = torch.where(p > 0, lp, 0.0)
    h = -(p * lp).sum(dim=1, keepdim=True)
    gl = torch.where(t < 0, 0.0, g_logp.double())[:, None]
    ge, gz = g_entropy.double()[:, None], g_lse.double()[:, None]
    one = torch.zeros_like(p)
    one.scatter_(1, t.clamp(min=0)[:, None], 1.0)
    size = gl.abs() * (one + p) + gz.abs() * p + ge.abs() * p * (lp.abs() + h)
    return gl * (one - p) + gz * p - ge * p * (lp + h), size, p, lp.abs(), h[:, 0]


def check_far(x, t, g, dx):
    """dx against exact_grad.  Up to |lse| = 64 the lse's rounding is 64 u of every
    p; beyond it p is formed from the row's sum again (r as above): in no row
    does the tolerance grow with |lse|."""
    V = x.shape[1]
    ref, size, p, lp, h = exact_grad(x, t, *g)
    r = (200 + V / 256 + 110) * U
    th = r * (100 + math.log(V)) / 10 + 4 * U * (h.abs() + 20)
    tz = r + 84 * U
    tol = (2 * tz + 4 * U * (lp.clamp(max=200) + 1) + 8 * U) * size
    tol = tol + p * (tz + th[:, None]) * g[1].double().abs()[:, None]
    tol = tol + (HB if x.dtype is torch.bfloat16 else U) * (ref.abs() + tol) + 1e-38
    close(dx, ref, tol, "gradient")


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("V", [40, 1001, 20003])
def test_gradient_of_logits_far_from_zero(cuda, V, dtype):
    """An offset of a row's logits, however large, changes p by no more than its
    own roundings; rows of one value, and of the type's lowest and largest."""
    log(f"logprobs: gradients of far logits {V} {dtype}")
    least, most = torch.finfo(dtype).min, torch.finfo(dtype).max
    base, _, _ = case(1, V, torch.float32, V)
    half = torch.arange(V) % 2 == 0
    rows = [base[0] + c for c in (0.0, 45.0, 52.0, 58.0, 70.0, -60.0, -90.0, 1e3, -1e3, 1e5, -1e5, 1e7,
                                  -1e7, 1e20, -1e30)]
    rows += [torch.full((V,), c) for c in (least, most, 80.0, -1e6)]
    rows += [torch.where(half, base[0] + 1e4, least), torch.where(half, base[0] - 1e4, float("-inf"))]
    one = torch.full((V,), least)
    one[V - 1] = most
    x = torch.stack(rows + [one]).to(dtype)
    n = len(x)
    gen = torch.Generator().manual_seed(V)
    t = torch.randint(0, V, (n,), generator=gen)
    t[::5] = -1
    g = [torch.randn(n, generator=gen) for _ in range(3)]
    xd, td, gd = x.to(cuda), t.to(cuda), [y.to(cuda) for y in g]
    _, h, lse = dd.logprobs(xd, td)
    dx = dd.logprobs_backward(xd, td, lse, h, *gd)
    check_far(x, t, g, dx)
    # each p by itself: no target, the gradient of the lse alone
    ones = torch.ones(n)
    p = dd.logprobs_backward(xd, torch.full_like(td, -1), lse, h, g_lse=ones.to(cuda))
    check_far(x, torch.full_like(t, -1), [0 * ones, 0 * ones, ones], p)
    # in place, several workgroups to a row
    wide = torch.zeros(n, V + 3, dtype=dtype, device=cuda)
    part = wide[:, 1:V + 1]
    part.copy_(xd)
    dd.logprobs_backward(part, td, lse, h, *gd, out=part)
    assert torch.equal(part, dx) and not wide[:, 0].any() and not wide[:, V + 1:].any()
    leaf = xd.clone().requires_grad_()
    logp, h, lse = dd.token_logprobs(leaf, td)
    (logp * gd[0] + h * gd[1] + lse * gd[2]).sum().backward()
    assert torch.equal(leaf.grad, dx)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("V", [700, 9000])
def test_gradient_of_a_target_out_of_range(cuda, V, dtype):
    """A target of V or more: NaN where the log probability has a gradient, in its
    row alone."""
    log(f"logprobs: gradient of targets out of range {V} {dtype}")
    x, _, g = case(5, V, dtype, 9)
    x[4] += 100
    t = torch.tensor([0, V, -1, 2 ** 40, V])
    xd, td, gd = x.to(cuda), t.to(cuda), [y.to(cuda) for y in g]
    logp, h, lse = dd.logprobs(xd, td)
    assert torch.equal(logp.isnan().cpu(), t >= V)
    dx = dd.logprobs_backward(xd, td, lse, h, *gd).cpu()
    assert dx[t >= V].isnan().all() and torch.isfinite(dx[t < V]).all()
    dx = dd.logprobs_backward(xd, td, lse, h, None, *gd[1:])
    check_far(x, torch.full_like(t, -1), [torch.zeros(5), *g[1:]], dx)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_large_entropy_gradients_of_masked_logits(cuda, dtype):
    log(f"logprobs: large entropy gradients {dtype}")
    x, t, _ = case(6, 3001, dtype, 12)
    mask = torch.rand(6, 3001, generator=torch.Generator().manual_seed(1)) < 0.5
    mask[torch.arange(6), t.clamp(min=0)] = False
    g = torch.tensor([1e9, -1e9, 1e20, -1e20, 3e30, 1.0])
    for value in (float("-inf"), torch.finfo(dtype).min, -1e30):
        y = x.masked_fill(mask, value)
        yd, td = y.to(cuda), t.to(cuda)
        _, h, lse = dd.logprobs(yd, td)
        dx = dd.logprobs_backward(yd, td, lse, h, g_entropy=g.to(cuda)).cpu()
        assert (dx[mask] == 0).all() and torch.isfinite(dx).all()
        check_far(y, t, [torch.zeros(6), g, torch.zeros(6)], dx)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("offset", [0.0, 90.0, -200.0])
def test_gradient_of_a_part_of_the_columns(cuda, offset, dtype):
    """A row's lse and entropy with some of its columns (a vocabulary in parts):
    the columns' share of the row's gradient, also where the lse lies far from
    zero.  Tolerance: the lse's own rounding, |lse| u of p, is in it twice."""
    log(f"logprobs: gradient of a part of the columns, offset {offset} {dtype}")
    V, cuts = 12000, [0, 500, 9500, 12000]
    x, _, g = case(6, V, dtype, 21)
    x = (x.float() + offset).to(dtype)
    none = torch.full((6,), -1)
    xd, nd, gd = x.to(cuda), none.to(cuda), [y.to(cuda) for y in g]
    _, h, lse = dd.logprobs(xd, nd)
    whole = dd.logprobs_backward(xd, nd, lse, h, None, *gd[1:])
    check_far(x, none, g, whole)
    parts = [dd.logprobs_backward(xd[:, a:b], nd, lse, h, None, *gd[1:])
             for a, b in zip(cuts, cuts[1:])]
    ref, size, p, lp, hr = exact_grad(x, none, torch.zeros(6), *g[1:])
    z = lse.double().cpu().abs()[:, None]
    tol = (2 * (200 + V / 256 + 194) * U + 2 * U * z + 4 * U * (lp.clamp(max=200) + 1)) * size
    tol = tol + (2 * U * z + 1e-4) * p * g[1].double().abs()[:, None]
    tol = tol + (HB if dtype is torch.bfloat16 else U) * (ref.abs() + tol) + 1e-38
    close(torch.cat(parts, dim=1), ref, tol, "parts")

"""GPU parity of the 8-bit operators (RMSNorm, rows as codes, int8 products,
weight gradients from codes) against their float64 definitions.

Tolerances, elementwise, from the roundings on the way (u = 2^-24 is the
fp32 rounding, 2^-8 the bf16 one, both relative to the value):

* h, codes, the scales of ``quantize`` and the values of ``dequantize`` are
  exact: equal to the definition.
* rstd: a sum of d squares of which a thread adds at most 32 and the rest is a
  tree of at most ten levels and 15 waves: 57 u of a positive sum, halved by
  the root, and four roundings after it: 34 u.  The norm's scales: two more.
* y: 2^-8 and 37 u.
* dx: 2^-8 of the result and (57 + 34 + 10) u of the magnitudes added.
* dw of the norm: 2^-8 and the depth of its sum (rows of a wave, waves,
  partial rows: below 128 at these sizes) u of the magnitudes.
* int8 products: the sum is exact; its conversion, two products and the
  residual's addition: 2^-8 and 4 u of the magnitudes.
* weight gradients: 2^-8 and T u of the magnitudes (a sum of T products), and
  relative L2 <= 3e-3 (the rounding of the result alone: 1.7e-3).
"""
import ctypes

import numpy as np
import pytest
import torch

from paper_2405_13226_amd import _lib, block_ops as ops

import int8_oracle as O
import int8_routes as routes
from int8_oracle import bf16, f64
from parity import log, rel_l2

pytestmark = pytest.mark.gpu
U, B = 2.0 ** -24, 2.0 ** -8
EPS = 1e-5

# every form of a row: a quarter or half of a wave, one wave of 1-4 chunks per
# lane, a workgroup of 256 with 1-4, one of 1024; whole and ragged, one row to
# several workgroups
ROWS = [(1, 1), (50, 128), (33, 129), (41, 250), (19, 256), (3, 7), (2, 8), (1, 64), (5, 100),
        (9, 512), (2, 520), (1, 2048), (700, 2048), (601, 1416), (513, 1000), (3, 1021), (515, 1029), (2, 2056), (7, 4100), (3, 5632),
        (2, 8192), (2, 8200), (3, 10001), (2, 16384)]


def close(got, ref, tol, what):
    got, ref = np.asarray(got, dtype=np.float64), np.asarray(ref, dtype=np.float64)
    assert got.shape == ref.shape, what
    off = np.abs(got - ref) - tol
    assert np.isfinite(got).all(), what
    assert (off <= 1e-37).all(), (what, float(off.max()), int((off > 0).sum()))


def norm_case(rows, d, seed, residual):
    x = bf16((rows, d), seed, 2.0)
    r = bf16((rows, d), seed + 1) if residual else None
    w = (1 + 0.2 * bf16((d,), seed + 2).float()).to(torch.bfloat16)
    return x, r, w, (O.add(x, r) if residual else x)


@pytest.mark.parametrize("residual", [False, True])
@pytest.mark.parametrize("rows,d", ROWS)
def test_rms_norm(cuda, rows, d, residual):
    log(f"rms_norm {rows} x {d} residual={residual}")
    x, r, w, h = norm_case(rows, d, rows + d, residual)
    rg = None if r is None else r.to(cuda)
    y, hg, rstd = ops.rms_norm(x.to(cuda), w.to(cuda), residual=rg, eps=EPS)
    assert torch.equal(hg.cpu(), h)
    ref = O.rstd(f64(h), EPS)
    close(rstd.cpu().numpy(), ref, 34 * U * ref, "rstd")
    want = f64(h) * ref[:, None] * f64(w)
    close(f64(y), want, (B + 37 * U) * np.abs(want), "y")
    codes, scales, hg, rstd8 = ops.rms_norm_int8(x.to(cuda), w.to(cuda), residual=rg, eps=EPS)
    assert torch.equal(hg.cpu(), h) and torch.equal(rstd8, rstd)
    q, top = O.codes(f64(h) * f64(w))
    assert np.array_equal(codes.cpu().numpy(), q)
    close(scales.cpu().numpy(), top * ref / 127, 36 * U * top * ref / 127, "scales")


@pytest.mark.parametrize("rows,d", ROWS)
def test_quantize_and_back(cuda, rows, d):
    log(f"quantize {rows} x {d}")
    x = bf16((rows, d), d)
    codes, scales = ops.quantize(x.to(cuda))
    q, top = O.codes(f64(x))
    assert np.array_equal(codes.cpu().numpy(), q)
    assert np.array_equal(scales.cpu().numpy(), top.astype(np.float32) / np.float32(127))
    back = ops.dequantize(codes, scales)
    want = (torch.from_numpy(q).float() * scales.cpu()[:, None]).to(torch.bfloat16)
    assert torch.equal(back.cpu(), want)


def test_codes_at_the_borders(cuda):
    # 127 z / 254 = z / 2: every odd z is on a border and goes to the even code
    z = torch.arange(-254, 255, dtype=torch.float32)
    rows = [z, z * 2.0 ** -40, z * 2.0 ** 100, z * 2.0 ** -135]  # the last holds subnormals
    # every bf16 value of the top eight binades, under maxima of all significands
    bits = torch.arange(0x3f80 - 8 * 128, 0x3f80, dtype=torch.int32).to(torch.int16)
    ladder = bits.view(torch.bfloat16).float()
    for k in range(128, 256, 7):
        rows.append(torch.cat([ladder, torch.tensor([k / 128.0])]))
    for i, row in enumerate(rows):
        x = row.to(torch.bfloat16)[None]
        codes, scales = ops.quantize(x.to(cuda))
        q, top = O.codes(f64(x))
        assert np.array_equal(codes.cpu().numpy(), q), i
        assert np.array_equal(scales.cpu().numpy(), top.astype(np.float32) / np.float32(127)), i


@pytest.mark.parametrize("d", [64, 1416, 5632])
def test_rows_that_are_zero_or_not_finite(cuda, d):
    x = bf16((7, d), 3)
    x[1] = 0
    x[2, d // 2] = float("nan")
    x[4, 0] = float("inf")
    x[5, d - 1] = -float("inf")
    bad = [2, 4, 5]
    w = torch.ones(d, dtype=torch.bfloat16)
    codes, scales = ops.quantize(x.to(cuda))
    c8, s8, _, _ = ops.rms_norm_int8(x.to(cuda), w.to(cuda), eps=EPS)
    good = [i for i in range(7) if i not in bad]
    for c, s in ((codes, scales), (c8, s8)):
        c, s = c.cpu(), s.cpu()
        assert torch.isnan(s[bad]).all() and not c[bad].any()
        assert s[1] == 0 and not c[1].any()
        assert torch.isfinite(s[good]).all()
        assert np.array_equal(c[good].numpy(), O.codes(f64(x[good]))[0])
        v = ops.dequantize(c.to(cuda), s.to(cuda)).float().cpu()
        assert torch.isnan(v[bad]).all() and torch.isfinite(v[good]).all()
    y, _, rstd = ops.rms_norm(x.to(cuda), w.to(cuda), eps=EPS)
    y = y.float().cpu()
    assert torch.isfinite(y[good]).all() and not y[1].any()
    assert abs(float(rstd[1]) * EPS ** 0.5 - 1) < 1e-6
    assert torch.isnan(y[2]).all()


@pytest.mark.parametrize("off", [1, 8])
def test_rows_of_wider_matrices(cuda, off):
    # column slices, aligned and not, and a longer output around the values
    rows, d, wide = 37, 1000, 1100
    x, r = bf16((rows, wide), 1).to(cuda), bf16((rows, wide + 8), 2).to(cuda)
    w = bf16((d,), 3).to(cuda)
    xs, rs = x[:, off:off + d], r[:, 2 * off:2 * off + d]
    a = ops.rms_norm_int8(xs, w, residual=rs)
    b = ops.rms_norm_int8(xs.contiguous(), w, residual=rs.contiguous())
    for s, t in zip(a, b):
        assert torch.equal(s, t)
    for s, t in zip(ops.rms_norm(xs, w, rs), ops.rms_norm(xs.contiguous(), w, rs.contiguous())):
        assert torch.equal(s, t)
    q, s = ops.quantize(xs)
    q2, s2 = ops.quantize(xs.contiguous())
    assert torch.equal(q, q2) and torch.equal(s, s2)
    out = torch.full((rows + 2, wide), 7.0, dtype=torch.bfloat16, device=cuda)
    into = out[1:-1, off:off + d]
    ops.dequantize(q, s, out=into)
    assert torch.equal(into, ops.dequantize(q, s))
    keep = torch.ones_like(out, dtype=torch.bool)
    keep[1:-1, off:off + d] = False
    assert (out[keep] == 7.0).all()


@pytest.mark.parametrize("dres", [False, True])
@pytest.mark.parametrize("rows,d", ROWS + [(5000, 64), (17000, 520), (33000, 128)])
def test_rms_norm_backward(cuda, rows, d, dres):
    log(f"rms_norm_backward {rows} x {d} dres={dres}")
    h, dy = bf16((rows, d), 5, 2.0), bf16((rows, d), 6)
    w = (1 + 0.2 * bf16((d,), 7).float()).to(torch.bfloat16)
    r = bf16((rows, d), 8) if dres else None
    rs = torch.from_numpy(O.rstd(f64(h), EPS)).float()
    dx, dw = ops.rms_norm_backward(h.to(cuda), w.to(cuda), rs.to(cuda), dy.to(cuda),
                                   None if r is None else r.to(cuda))
    rx, rw, mag = O.norm_backward(f64(h), f64(w), f64(rs), f64(dy), None if r is None else f64(r))
    close(f64(dx), rx, B * np.abs(rx) + 101 * U * mag, "dx")
    sums = np.abs(f64(dy) * f64(h) * f64(rs)[:, None]).sum(0)
    close(f64(dw), rw, B * np.abs(rw) + 128 * U * sums, "dw")


def test_rms_norm_backward_is_the_gradient(cuda):
    # against differences of the norm itself in float64
    rows, d = 3, 40
    x, w, dy = (f64(bf16(s, i)) for i, s in enumerate([(rows, d), (d,), (rows, d)]))
    w = f64(round_to_bf16(1 + 0.1 * w))
    f = lambda x, w: (dy * (x * O.rstd(x, EPS)[:, None] * w)).sum()
    t = lambda a: torch.from_numpy(a).to(torch.bfloat16).to(cuda)
    rs = torch.from_numpy(O.rstd(x, EPS)).float().to(cuda)
    dx, dw = ops.rms_norm_backward(t(x), t(w), rs, t(dy))
    e = 1e-5
    for i, j in [(0, 0), (1, 7), (2, 39)]:
        p, m = x.copy(), x.copy()
        p[i, j] += e
        m[i, j] -= e
        num = (f(p, w) - f(m, w)) / (2 * e)
        # the difference: e^2 times a third derivative of order one
        assert abs(f64(dx)[i, j] - num) <= B * abs(num) + 1e-5
        p, m = w.copy(), w.copy()
        p[j] += e
        m[j] -= e
        num = (f(x, p) - f(x, m)) / (2 * e)
        assert abs(f64(dw)[j] - num) <= B * abs(num) + 1e-5


def round_to_bf16(a):
    return torch.from_numpy(a).to(torch.bfloat16)


def random_codes(rows, d, seed, dev, full=False):
    g = torch.Generator(device="cpu").manual_seed(seed)
    q = torch.randint(-128 if full else -127, 128, (rows, d), generator=g).to(torch.int8)
    s = torch.rand(rows, generator=g) * 0.02 + 1e-3
    return q.to(dev), s.to(dev)


def check_product(q, s, p, t, r, c):
    ref = O.product(q.cpu().numpy(), f64(s), p.cpu().numpy(), f64(t))
    mag = np.abs(ref)
    if r is not None:
        ref, mag = ref + f64(r), mag + np.abs(f64(r))
    close(f64(c), ref, B * np.abs(ref) + 4 * U * mag, "c")


SIZES = [(1, 1, 16), (1, 48, 64), (1, 1000, 2048), (2, 17, 80), (3, 5, 16), (5, 300, 1040),
         (16, 64, 128), (16, 2000, 2048), (17, 33, 48), (31, 640, 512), (33, 257, 4096),
         (64, 64, 64), (64, 1000, 528), (65, 63, 144), (100, 128, 128), (127, 129, 256),
         (128, 128, 272), (200, 500, 1040), (257, 255, 384), (300, 1029, 1808), (512, 512, 2048),
         (1000, 130, 96), (1531, 777, 640), (2, 9000, 16), (2300, 2600, 128), (2304, 4352, 400)]


@pytest.mark.parametrize("residual", [False, True])
@pytest.mark.parametrize("M,N,K", SIZES)
def test_gemm_int8(cuda, M, N, K, residual):
    log(f"gemm_int8 M={M} N={N} K={K} residual={residual}")
    q, s = random_codes(M, K, M + K, cuda, full=True)
    p, t = random_codes(N, K, N + K + 1, cuda, full=True)
    r = bf16((M, N), 9, 3.0).to(cuda) if residual else None
    c = ops.gemm_int8(q, s, p, t, residual=r)
    check_product(q, s, p, t, r, c)


# The large tiles' workgroups walk several tiles as one sequence of steps: one
# step a tile to several, odd counts (whose tiles start in alternating stages),
# whole and ragged tiles, with and without stores that waits must pass over.
@pytest.mark.parametrize("residual", [False, True])
@pytest.mark.parametrize("K", [16, 128, 144, 272, 400, 640, 1040])
@pytest.mark.parametrize("M,N", [(16384, 12288), (16400, 12289)])
def test_gemm_int8_several_tiles_a_workgroup(cuda, M, N, K, residual):
    assert routes.product(M, N, K) == "large"
    q, s = random_codes(M, K, M + K, cuda, full=True)
    p, t = random_codes(N, K, N + K + 1, cuda, full=True)
    gen = torch.Generator(device=cuda).manual_seed(K)
    r = torch.randn((M, N), generator=gen, device=cuda).to(torch.bfloat16) if residual else None
    c = ops.gemm_int8(q, s, p, t, residual=r)
    rows = np.unique(np.r_[np.random.default_rng(0).choice(M, 100, replace=False), 0, 255, 256,
                           M - 1])
    check_product(q[rows], s[rows], p, t, None if r is None else r[rows], c[rows])
    # every other element against the small tiles, whose sums are the same
    for m in range(0, M, 2100):
        assert routes.product(min(2100, M - m), 4000, K) == "small"
        for n in range(0, N, 4000):
            part = ops.gemm_int8(q[m:m + 2100], s[m:m + 2100].contiguous(), p[n:n + 4000],
                                 t[n:n + 4000].contiguous(),
                                 residual=None if r is None else
                                 r[m:m + 2100, n:n + 4000].contiguous())
            assert torch.equal(c[m:m + 2100, n:n + 4000], part)


def test_gemm_int8_more_tiles_a_workgroup_than_lanes(cuda):
    M, N, K = 65536, 16650, 48
    assert routes.product(M, N, K) == "large" and 256 * ((N + 255) // 256) > 64 * routes.CUS
    q, s = random_codes(M, K, 1, cuda)
    p, t = random_codes(N, K, 2, cuda)
    c = ops.gemm_int8(q, s, p, t)
    rows = np.unique(np.r_[np.arange(0, M, 509), M - 1])
    check_product(q[rows], s[rows], p, t, None, c[rows])


@pytest.mark.parametrize("M,N,K,form", [(64, 300, 80, "few"), (65, 300, 80, "small"),
                                        (1531, 777, 640, "small"), (2048, 6144, 2048, "large"), (9000, 6152, 912, "large")])
def test_products_reach_every_form(cuda, M, N, K, form):
    assert routes.product(M, N, K) == form
    q, s = random_codes(M, K, 3, cuda)
    p, t = random_codes(N, K, 4, cuda)
    check_product(q, s, p, t, None, ops.gemm_int8(q, s, p, t))


def test_gemm_int8_extreme_codes_sum_exactly(cuda):
    # all codes -128: the longest sum is 131056 * 2^14, just below 2^31
    for M, N in ((1, 20), (70, 70)):
        K = (1 << 17) - 16
        q = torch.full((M, K), -128, dtype=torch.int8, device=cuda)
        p = torch.full((N, K), -128, dtype=torch.int8, device=cuda)
        one = torch.ones(max(M, N), device=cuda)
        c = ops.gemm_int8(q, one[:M].contiguous(), p, one[:N].contiguous())
        want = torch.tensor(float(K * 128 * 128)).to(torch.bfloat16).float()
        assert (c.float().cpu() == want).all()


@pytest.mark.parametrize("M,N,K", [(1, 100, 256), (40, 100, 272), (300, 264, 400)])
def test_gemm_int8_strided_and_in_place(cuda, M, N, K):
    q, s = random_codes(M, K + 48, 1, cuda)
    p, t = random_codes(N, K + 32, 2, cuda)
    qs, ps = q[:, 16:16 + K], p[:, 32:32 + K]
    want = ops.gemm_int8(qs.contiguous(), s, ps.contiguous(), t)
    for off in (0, 1, 8):
        out = torch.full((M + 2, N + 24), 5.0, dtype=torch.bfloat16, device=cuda)
        into = out[1:-1, off:off + N]
        ops.gemm_int8(qs, s, ps, t, out=into)
        assert torch.equal(into, want)
        keep = torch.ones_like(out, dtype=torch.bool)
        keep[1:-1, off:off + N] = False
        assert (out[keep] == 5.0).all()
        r = bf16((M, N), 4).to(cuda)
        into.copy_(r)
        ops.gemm_int8(qs, s, ps, t, residual=into, out=into)
        assert torch.equal(into, ops.gemm_int8(qs, s, ps, t, residual=r))
        assert (out[keep] == 5.0).all()


def test_gemm_int8_scales_that_are_not_finite(cuda):
    # a poisoned token poisons its row, a zero one gives the residual
    M, N, K = 70, 90, 128
    q, s = random_codes(M, K, 1, cuda)
    p, t = random_codes(N, K, 2, cuda)
    r = bf16((M, N), 3).to(cuda)
    clean = ops.gemm_int8(q, s, p, t, residual=r)
    s2 = s.clone()
    s2[5], s2[66] = float("nan"), 0.0
    c = ops.gemm_int8(q, s2, p, t, residual=r)
    assert torch.isnan(c[5]).all() and torch.equal(c[66], r[66])
    others = [i for i in range(M) if i not in (5, 66)]
    assert torch.equal(c[others], clean[others])


WGRAD = [(1, 8, 8), (2, 16, 40), (63, 64, 64), (64, 72, 128), (65, 128, 72), (200, 256, 256),
         (129, 264, 520), (1000, 520, 264), (3001, 1040, 1416), (64, 512, 768), (192, 256, 512),
         (4096, 256, 256), (8200, 512, 264), (300, 2304, 2560), (20000, 136, 200),
         (8192, 1024, 1416), (4100, 2056, 1000), (700, 4352, 4360), (9000, 1800, 5000)]


@pytest.mark.parametrize("T,M,N", WGRAD)
def test_gemm_int8_wgrad(cuda, T, M, N):
    log(f"gemm_int8_wgrad T={T} M={M} N={N}")
    q, s = random_codes(T, M, T + M, cuda)
    dy = bf16((T, N), N).to(cuda)
    dw = ops.gemm_int8_wgrad(q, s, dy)
    x = f64(ops.dequantize(q, s))
    ref = x.T @ f64(dy)
    mag = np.abs(x).T @ np.abs(f64(dy))
    close(f64(dw), ref, B * np.abs(ref) + T * U * mag, "dw")
    assert rel_l2(f64(dw), ref) <= 3e-3


@pytest.mark.parametrize("T,M,N,edge,shared", [
    (1000, 520, 264, 128, False), (4096, 1024, 1024, 128, True), (16384, 2048, 2048, 256, True),
    (1024, 4096, 4096, 256, False), (2048, 4200, 4360, 256, True)])
def test_weight_gradients_reach_every_form(cuda, T, M, N, edge, shared):
    form = routes.wgrad(T, M, N)
    assert form["edge"] == edge and (form["shared"] > 0) == shared, form
    q, s = random_codes(T, M, 5, cuda)
    dy = bf16((T, N), 6).to(cuda)
    dw = f64(ops.gemm_int8_wgrad(q, s, dy))
    x = f64(ops.dequantize(q, s))
    rows = np.unique(np.r_[np.random.default_rng(0).choice(M, 100, replace=False), 0, M - 1])
    ref = x[:, rows].T @ f64(dy)
    mag = np.abs(x[:, rows]).T @ np.abs(f64(dy))
    close(dw[rows], ref, B * np.abs(ref) + T * U * mag, "dw")
    assert rel_l2(dw[rows], ref) <= 3e-3


@pytest.mark.parametrize("T,M,N", [(100, 40, 72), (500, 264, 264)])
def test_gemm_int8_wgrad_strided(cuda, T, M, N):
    q, s = random_codes(T, M + 24, 1, cuda)
    dy = bf16((T, N + 16), 2).to(cuda)
    want = ops.gemm_int8_wgrad(q[:, 8:8 + M].contiguous(), s, dy[:, 8:8 + N].contiguous())
    out = torch.full((M + 2, N + 24), 5.0, dtype=torch.bfloat16, device=cuda)
    into = out[1:-1, 8:8 + N]
    ops.gemm_int8_wgrad(q[:, 8:8 + M], s, dy[:, 8:8 + N], out=into)
    assert torch.equal(into, want)
    keep = torch.ones_like(out, dtype=torch.bool)
    keep[1:-1, 8:8 + N] = False
    assert (out[keep] == 5.0).all()


@pytest.mark.parametrize("n", [1, 2, 3])
@pytest.mark.parametrize("T,M,N", [(100, 40, 72), (2000, 520, 264), (4096, 1024, 1024),
                                   (2048, 2048, 2816)])
def test_gemm_int8_wgrad_group(cuda, T, M, N, n):
    # gradients of one input together, into column slices of one matrix
    q, s = random_codes(T, M, T, cuda)
    dys = [bf16((T, N), 10 + i).to(cuda) for i in range(n)]
    dw = torch.full((M, n * N), 5.0, dtype=torch.bfloat16, device=cuda)
    columns = [dw[:, i * N:(i + 1) * N] for i in range(n)]
    ops.gemm_int8_wgrad_group(q, s, dys, outs=columns)
    x = f64(ops.dequantize(q, s))
    for i in range(n):
        ref = x.T @ f64(dys[i])
        close(f64(columns[i]), ref, B * np.abs(ref) + T * U * (np.abs(x).T @ np.abs(f64(dys[i]))),
              i)
    for a, b in zip(ops.gemm_int8_wgrad_group(q, s, dys), columns):
        assert torch.equal(a, b)


def test_gemm_int8_wgrad_rows_behind_the_last_token(cuda):
    # what lies behind the last token is not read into the sums
    T, M, N = 70, 264, 520
    q, s = random_codes(T + 60, M, 1, cuda)
    dy = bf16((T + 60, N), 2).to(cuda)
    want = ops.gemm_int8_wgrad(q[:T].clone(), s[:T].clone(), dy[:T].clone())
    dy[T:] = float("nan")
    s[T:] = float("inf")
    assert torch.equal(ops.gemm_int8_wgrad(q[:T], s[:T].contiguous(), dy[:T]), want)


def test_offsets_past_32_bits(cuda):
    # 2.3e9 elements: the last rows are those of a matrix of their own
    rows, d = 280_000, 8192
    assert rows * d > 2 ** 31
    x = torch.empty((rows, d), dtype=torch.bfloat16, device=cuda)
    tail = bf16((64, d), 1).to(cuda)
    x.zero_()
    x[-64:] = tail
    w = (1 + 0.1 * bf16((d,), 2).float()).to(torch.bfloat16).to(cuda)
    q, s = ops.quantize(x)
    q1, s1 = ops.quantize(tail)
    assert torch.equal(q[-64:], q1) and torch.equal(s[-64:], s1) and not s[:-64].any()
    assert torch.equal(ops.dequantize(q, s)[-64:], ops.dequantize(q1, s1))
    dw = ops.gemm_int8_wgrad(q, s, torch.ones((rows, 8), dtype=torch.bfloat16, device=cuda))
    ref = f64(ops.dequantize(q1, s1)).sum(0)
    mag = np.abs(f64(ops.dequantize(q1, s1))).sum(0)
    close(f64(dw)[:, 0], ref, B * np.abs(ref) + 64 * U * mag, "dw")
    del q
    for a, b in zip(ops.rms_norm(x, w, residual=x), ops.rms_norm(tail, w, residual=tail)):
        assert torch.equal(a[-64:], b)
    r = torch.ones(rows, device=cuda)
    dx, _ = ops.rms_norm_backward(x, w, r, x)
    assert torch.equal(dx[-64:], ops.rms_norm_backward(tail, w, r[:64].contiguous(), tail)[0])


@pytest.mark.parametrize("M,N", [(70_000, 32_768), (8_400_000, 264)])
def test_products_past_32_bits(cuda, M, N):
    assert M * N > 2 ** 31
    q, s = random_codes(M, 32, 1, cuda)
    p, t = random_codes(N, 32, 2, cuda)
    c = ops.gemm_int8(q, s, p, t)
    rows = np.r_[0:8, M // 2:M // 2 + 8, M - 8:M]
    check_product(q[rows], s[rows], p, t, None, c[rows])


def test_product_of_one_token_with_more_channels_than_a_grid_of_few_tokens_holds(cuda):
    N = 32 * (1 << 23) + 40
    p = torch.ones((N, 16), dtype=torch.int8, device=cuda)
    p[-1], p[0] = 2, 3
    q = torch.ones((1, 16), dtype=torch.int8, device=cuda)
    one = torch.ones(1, device=cuda)
    c = ops.gemm_int8(q, one, p, torch.ones(N, device=cuda))
    assert c[0, 0] == 48 and c[0, -1] == 32 and bool((c[0, 1:-1] == 16).all())


@pytest.mark.parametrize("d", [8, 2048])
def test_norm_of_a_row_whose_squares_overflow_fp32_is_zero(cuda, d):
    x = torch.ones((3, d), dtype=torch.bfloat16, device=cuda)
    x[1] = 2e19  # its square alone is 4e38, past fp32
    w = torch.ones(d, dtype=torch.bfloat16, device=cuda)
    y, h, rstd = ops.rms_norm(x, w)
    assert rstd[1] == 0 and not y[1].any() and torch.equal(h, x)
    assert bool((y[0] == 1).all()) and bool((y[2] == 1).all())
    q, s, _, rstd = ops.rms_norm_int8(x, w)
    assert rstd[1] == 0 and s[1] == 0 and not ops.dequantize(q, s)[1].any()
    dx, dw = ops.rms_norm_backward(x, w, rstd, torch.ones_like(x))
    assert not dx[1].any() and bool(dw.isfinite().all())


def test_empty_matrices(cuda):
    e = lambda *s, t=torch.bfloat16: torch.empty(s, dtype=t, device=cuda)
    y, h, rstd = ops.rms_norm(e(0, 64), e(64))
    assert y.shape == (0, 64) and rstd.shape == (0,)
    assert ops.rms_norm_int8(e(0, 64), e(64))[0].shape == (0, 64)
    dx, dw = ops.rms_norm_backward(e(0, 64), e(64), e(0, t=torch.float32), e(0, 64))
    assert dx.shape == (0, 64) and not dw.any()
    q, s = ops.quantize(e(0, 64))
    assert ops.dequantize(q, s).shape == (0, 64)
    b, sb = ops.quantize(e(32, 64).zero_())
    assert ops.gemm_int8(q, s, b, sb).shape == (0, 32)
    q0, s0 = ops.quantize(e(4, 0))
    assert q0.shape == (4, 0) and not s0.any()
    dw = ops.gemm_int8_wgrad(q, s, e(0, 16))
    assert dw.shape == (64, 16) and not dw.any()
    assert ops.gemm_int8_wgrad(b[:, :0].contiguous(), sb, e(32, 16)).shape == (0, 16)


def layer_step(x, r, nw, w8, sw, w, dy, dh):
    """A linear layer behind the norm, forward in 8 bits, and its backward
    from the codes it kept."""
    q, s, h, rstd = ops.rms_norm_int8(x, nw, residual=r)
    y = ops.gemm_int8(q, s, w8, sw)
    dw = ops.gemm_int8_wgrad(q, s, dy)
    da = ops.gemm(dy, w, trans_b=True)
    dx, dnw = ops.rms_norm_backward(h, nw, rstd, da, dres=dh)
    return y, dw, dx, dnw


def layer_inputs(T, d, n, dev):
    x, r, dy, dh = bf16((T, d), 1), bf16((T, d), 2), bf16((T, n), 3), bf16((T, d), 4)
    nw, w = (1 + 0.1 * bf16((d,), 5).float()).to(torch.bfloat16), bf16((d, n), 6, 0.05)
    w8, sw = ops.quantize(w.t().contiguous().to(dev))
    return [t.to(dev) for t in (x, r, nw)] + [w8, sw] + [t.to(dev) for t in (w, dy, dh)]


def test_layer_forward_and_backward_together(cuda):
    T, d, n = 512, 768, 1024
    args = layer_inputs(T, d, n, cuda)
    x, r, nw, w8, sw, w, dy, dh = args
    y, dw, dx, dnw = layer_step(*args)
    h = f64(O.add(x.cpu(), r.cpu()))
    rs = O.rstd(h, ops.LN_EPS)
    q, top = O.codes(h * f64(nw))
    a = q * (top * rs / 127)[:, None]
    # one bf16 rounding of each result (1.7e-3); dw also rounds its restored
    # input, dx and dnw the gradient between the two products
    assert rel_l2(f64(y), a @ (w8.cpu().numpy() * f64(sw)[:, None]).T) <= 3e-3
    assert rel_l2(f64(dw), a.T @ f64(dy)) <= 5e-3
    rx, rnw, _ = O.norm_backward(h, f64(nw), rs, f64(dy) @ f64(w).T, f64(dh))
    assert rel_l2(f64(dx), rx) <= 5e-3 and rel_l2(f64(dnw), rnw) <= 5e-3
    # and the 8-bit layer is the bf16 one up to its codes: each operand is off
    # by up to half a step of A / 127 with A about four deviations, 0.9% of a
    # deviation (rms), the two together 1.3%
    plain = (h * rs[:, None] * f64(nw)) @ f64(w)
    assert rel_l2(f64(y), plain) <= 2e-2


def test_repeated_calls_are_bit_identical(cuda):
    args = layer_inputs(768, 512, 768, cuda)
    first = layer_step(*args)
    for _ in range(2):
        for a, b in zip(layer_step(*args), first):
            assert torch.equal(a, b)


def test_on_another_stream(cuda):
    args = layer_inputs(256, 256, 512, cuda)
    ref = layer_step(*args)
    torch.cuda.synchronize()
    side = torch.cuda.Stream(cuda)
    with torch.cuda.stream(side):
        out = layer_step(*args)
    side.synchronize()
    for a, b in zip(out, ref):
        assert torch.equal(a, b)


@pytest.mark.parametrize("T,d,n", [(256, 256, 512), (2048, 1024, 2816)])
def test_graph_replay_matches_eager(cuda, T, d, n):
    args = layer_inputs(T, d, n, cuda)
    one = [args[0][:1], args[1][:1]] + args[2:5]  # and the single-token form

    def step():
        q, s, h, _ = ops.rms_norm_int8(one[0], one[2], residual=one[1])
        return layer_step(*args) + (ops.gemm_int8(q, s, one[3], one[4]), h)

    ref = [t.clone() for t in step()]
    torch.cuda.synchronize()
    side = torch.cuda.Stream(cuda)
    side.wait_stream(torch.cuda.current_stream(cuda))
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream(cuda).wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        out = step()
    other = layer_inputs(256, 512, 256, cuda)
    for rep in range(3):
        for t in out:
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        for i, (a, b) in enumerate(zip(out, ref)):
            assert torch.equal(a, b), (rep, i)
        layer_step(*other)
        torch.cuda.synchronize()


def test_two_streams_at_once(cuda):
    # Equal sizes, other values: what one call left where the other reads shows.
    cases = [layer_inputs(2048, 1024, 2816, cuda), layer_inputs(2048, 1024, 2816, cuda)]
    cases[1][0] = cases[1][0] * 3
    ref = [[t.clone() for t in layer_step(*c)] for c in cases]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(cuda) for _ in cases]
    out = [[], []]
    for _ in range(4):
        for i, st in enumerate(streams):
            with torch.cuda.stream(st):
                out[i].append(layer_step(*cases[i]))
    torch.cuda.synchronize()
    for i in range(2):
        for step in out[i]:
            for a, b in zip(step, ref[i]):
                assert torch.equal(a, b), i


def test_two_graphs_at_once(cuda):
    cases = [layer_inputs(2048, 1024, 2816, cuda), layer_inputs(2048, 1024, 2816, cuda)]
    cases[1][0] = cases[1][0] * 3
    ref = [[t.clone() for t in layer_step(*c)] for c in cases]
    torch.cuda.synchronize()
    graphs, outs = [], []
    streams = [torch.cuda.Stream(cuda) for _ in cases]
    for c, st in zip(cases, streams):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=st):
            outs.append(layer_step(*c))
        graphs.append(g)
    for rep in range(3):
        for g, st in zip(graphs, streams):
            with torch.cuda.stream(st):
                g.replay()
        torch.cuda.synchronize()
        for i in range(2):
            for a, b in zip(outs[i], ref[i]):
                assert torch.equal(a, b), (rep, i)
                a.zero_()
        torch.cuda.synchronize()


def test_the_same_tensor_twice(cuda):
    q, s = ops.quantize(bf16((300, 512), 5).to(cuda))
    assert torch.equal(ops.gemm_int8(q, s, q, s),
                       ops.gemm_int8(q, s, q.clone(), s.clone()))
    dy = bf16((300, 264), 6).to(cuda)
    one = ops.gemm_int8_wgrad_group(q, s, [dy, dy.clone(), dy.clone()])
    for a, b in zip(ops.gemm_int8_wgrad_group(q, s, [dy, dy, dy]), one):
        assert torch.equal(a, b)
    x = bf16((40, 512), 7).to(cuda)
    w = torch.ones(512, dtype=torch.bfloat16, device=cuda)
    for a, b in zip(ops.rms_norm(x, w, residual=x), ops.rms_norm(x, w, residual=x.clone())):
        assert torch.equal(a, b)


class Guarded:
    """A tensor of this shape inside a buffer with bands of a pattern around it."""

    def __init__(self, shape, dtype, dev):
        n = int(np.prod(shape)) * torch.empty(0, dtype=dtype).element_size()
        self.raw = torch.full((4096 + n + 4096,), 0xA5, dtype=torch.uint8, device=dev)
        self.t = self.raw[4096:4096 + n].view(dtype).view(shape)
        self.p = ctypes.c_void_p(self.t.data_ptr())

    def intact(self):
        n = self.raw.numel()
        return bool((self.raw[:4096] == 0xA5).all() and (self.raw[n - 4096:] == 0xA5).all())


def at(t):
    return ctypes.c_void_p(t.data_ptr())


@pytest.mark.parametrize("rows,d", [(7, 1), (33, 100), (19, 256), (5, 1021), (700, 1032), (3, 8200)])
def test_row_outputs_stay_inside_their_buffers(cuda, rows, d):
    lib, st = _lib.lib(), ctypes.c_void_p(torch.cuda.current_stream().cuda_stream)
    G = lambda *shape, dtype=torch.bfloat16: Guarded(shape, dtype, cuda)
    x, r, dy = (bf16((rows, d), i).to(cuda) for i in range(3))
    w = bf16((d,), 4).to(cuda)
    f32, i8 = torch.float32, torch.int8
    h, y, rstd = G(rows, d), G(rows, d), G(rows, dtype=f32)
    assert lib.dd_rmsnorm_fwd(at(x), d, at(r), d, at(w), h.p, y.p, rstd.p, rows, d, 1e-5, st) == 0
    h8, q, s, rstd8 = G(rows, d), G(rows, d, dtype=i8), G(rows, dtype=f32), G(rows, dtype=f32)
    assert lib.dd_rmsnorm_int8_fwd(at(x), d, at(r), d, at(w), h8.p, q.p, d, s.p, rstd8.p, rows, d,
                                   1e-5, st) == 0
    need = lib.dd_rmsnorm_bwd_workspace_bytes(rows, d)
    dx, dw, ws = G(rows, d), G(d), G(need, dtype=torch.uint8)
    assert lib.dd_rmsnorm_bwd(h.p, at(w), rstd.p, at(dy), at(r), dx.p, dw.p, rows, d, ws.p, need,
                              st) == 0
    q2, s2, v = G(rows, d, dtype=i8), G(rows, dtype=f32), G(rows, d)
    assert lib.dd_quantize(at(x), d, q2.p, d, s2.p, rows, d, st) == 0
    assert lib.dd_dequantize(q2.p, d, s2.p, v.p, d, rows, d, st) == 0
    torch.cuda.synchronize()
    for i, g in enumerate((h, y, rstd, h8, q, s, rstd8, dx, dw, ws, q2, s2, v)):
        assert g.intact(), i
    assert torch.equal(h.t, h8.t) and torch.isfinite(dx.t.float()).all()


@pytest.mark.parametrize("M,N,K", [(1, 1, 16), (33, 77, 48), (130, 257, 80), (2300, 2601, 144),
                                   (9001, 6153, 912)])
def test_products_stay_inside_their_buffers(cuda, M, N, K):
    lib, st = _lib.lib(), ctypes.c_void_p(torch.cuda.current_stream().cuda_stream)
    q, s = random_codes(M, K, 1, cuda)
    p, t = random_codes(N, K, 2, cuda)
    c = Guarded((M, N), torch.bfloat16, cuda)
    assert lib.dd_gemm_i8(at(q), K, at(s), at(p), K, at(t), None, c.p, N, M, N, K, st) == 0
    torch.cuda.synchronize()
    assert c.intact() and torch.isfinite(c.t.float()).all()


@pytest.mark.parametrize("T,M,N,n", [(1, 8, 8, 1), (70, 136, 264, 2), (1300, 264, 136, 3),
                                     (5000, 1096, 2704, 1), (20000, 136, 200, 1),
                                     (9000, 1032, 2824, 1)])
def test_weight_gradients_stay_inside_their_buffers(cuda, T, M, N, n):
    lib, st = _lib.lib(), ctypes.c_void_p(torch.cuda.current_stream().cuda_stream)
    q, s = random_codes(T, M, 1, cuda)
    dys = [bf16((T, N), 2 + i).to(cuda) for i in range(n)]
    need = lib.dd_gemm_i8_wgrad_workspace_bytes(T, M, N, n)
    dws = [Guarded((M, N), torch.bfloat16, cuda) for _ in range(n)]
    ws = Guarded((need,), torch.uint8, cuda)
    ptrs = lambda ps: (ctypes.c_void_p * n)(*ps)
    assert lib.dd_gemm_i8_wgrad(at(q), M, at(s), ptrs([y.data_ptr() for y in dys]), N,
                                ptrs([w.t.data_ptr() for w in dws]), N, n, T, M, N, ws.p, need,
                                st) == 0
    torch.cuda.synchronize()
    assert ws.intact()
    for w, y in zip(dws, dys):
        assert w.intact() and torch.equal(w.t, ops.gemm_int8_wgrad_group(q, s, dys)[dws.index(w)])


def extreme_rows(d, seed):
    """Rows of every magnitude that bf16 has, one of zeros, two not finite."""
    x = torch.stack([bf16((d,), seed + i).double() * 2.0 ** e
                     for i, e in enumerate((-128, -100, -62, -30, 0, 30, 60, 100, 125))])
    x = x.clamp(-3e38, 3e38).to(torch.bfloat16)
    bad = torch.stack([x[4].clone(), x[0].clone(), torch.zeros_like(x[0])])
    bad[0, d // 2], bad[1, d - 1] = float("nan"), float("inf")
    return torch.cat([x, bad])


@pytest.mark.parametrize("weight", [-126, -70, 0, 65, 120, "mixed"])
@pytest.mark.parametrize("residual", [False, True])
@pytest.mark.parametrize("d", [7, 250, 1416, 2056, 8200])
def test_norm_codes_whose_products_leave_fp32(cuda, d, residual, weight):
    # h w passes 3.4e38 or loses bits below 2^-126: its codes are the nearest
    # ones all the same, and its scale has rstd's magnitude back
    x = extreme_rows(d, d)
    r = extreme_rows(d, d + 50) if residual else None
    w = bf16((d,), 3).double()
    w = w * (2.0 ** torch.linspace(-120, 120, d).double() if weight == "mixed" else 2.0 ** weight)
    w = w.clamp(-3e38, 3e38).to(torch.bfloat16)
    h = x if r is None else O.add(x, r)
    q, s, hg, rstd = ops.rms_norm_int8(x.to(cuda), w.to(cuda),
                                       residual=None if r is None else r.to(cuda), eps=EPS)
    bad = ~torch.isfinite(h.float()).all(1).numpy()
    assert bad.sum() >= 2
    q, s, rstd = q.cpu().numpy(), s.double().cpu().numpy(), rstd.double().cpu().numpy()
    want, top = O.codes(f64(h) * f64(w))
    assert np.isnan(s[bad]).all() and not q[bad].any()
    good = ~bad
    ref = O.rstd(f64(h)[good], EPS)
    over = (f64(h)[good] ** 2).sum(1) > 3.4e38  # documented: such rows give zeros
    assert over.any() and (s[good][over] == 0).all() and (rstd[good][over] == 0).all()
    assert np.array_equal(q[good], want[good])
    scale = np.where(over, 0, top[good] * ref / 127)
    assert (scale < 3.4e38).all()
    # 2^-150: half a step of an fp32 scale below 2^-126
    assert (np.abs(s[good] - scale) <= 36 * U * scale + 2.0 ** -150).all()


def test_norm_codes_of_extreme_rows_among_others_of_a_workgroup(cuda):
    # more rows than the grid has workgroups: a workgroup's second row reuses
    # what its first one reduced through
    rows, d, grid = (1 << 20) + 512, 2056, 1 << 20
    x = torch.ones((rows, d), dtype=torch.bfloat16, device=cuda)
    block = bf16((512, d), 1).to(cuda)
    x[:512], x[grid:] = block, block.flip(0)
    w = (1 + 0.1 * bf16((d,), 2).float()).to(torch.bfloat16).to(cuda)
    x[0:512:3] *= 2.0 ** -100
    x[1:512:3] = 0
    x[grid + 1::2] *= 2.0 ** -110
    q, s, _, rstd = ops.rms_norm_int8(x, w)
    for part in (slice(0, 512), slice(grid, rows)):
        for a, b in zip(ops.rms_norm_int8(x[part].contiguous(), w), (q[part], s[part], x[part],
                                                                     rstd[part])):
            assert torch.equal(a, b)
        want, _ = O.codes(f64(x[part]) * f64(w))
        assert np.array_equal(q[part].cpu().numpy(), want)
    assert torch.equal(s[512:grid].min(), s[512:grid].max())


@pytest.mark.parametrize("d", [7, 100, 256, 1021, 2048, 4104, 10001])
def test_norm_codes_of_zero_and_extreme_rows_in_wider_matrices(cuda, d):
    # rows inside wider ones on all sides: what is beside them stays as it was
    lib, st = _lib.lib(), ctypes.c_void_p(torch.cuda.current_stream().cuda_stream)
    x, r = extreme_rows(d, 1), extreme_rows(d, 60)
    x[3], r[3] = 0, 0
    x[5], r[5] = bf16((d,), 9), -bf16((d,), 9)  # a sum of zeros
    rows, wide = x.shape[0], d + 24
    w = (1 + 0.1 * bf16((d,), 2).float()).to(torch.bfloat16).to(cuda)
    xw, rw = (torch.full((rows, wide), 3.0, dtype=torch.bfloat16, device=cuda) for _ in range(2))
    xw[:, 5:5 + d], rw[:, 1:1 + d] = x.to(cuda), r.to(cuda)
    q = torch.full((rows + 2, wide), 77, dtype=torch.int8, device=cuda)
    h, s, rstd = (Guarded(shape, t, cuda) for shape, t in (((rows, d), torch.bfloat16),
                                                           ((rows,), torch.float32),
                                                           ((rows,), torch.float32)))
    into = q[1:-1, 3:3 + d]
    assert lib.dd_rmsnorm_int8_fwd(at(xw[:, 5:]), wide, at(rw[:, 1:]), wide, at(w), h.p, at(into),
                                   wide, s.p, rstd.p, rows, d, 1e-5, st) == 0
    torch.cuda.synchronize()
    keep = torch.ones_like(q, dtype=torch.bool)
    keep[1:-1, 3:3 + d] = False
    assert bool((q[keep] == 77).all()) and all(g.intact() for g in (h, s, rstd))
    sums = O.add(x, r)
    want, top = O.codes(f64(sums) * f64(w))
    assert np.array_equal(into.cpu().numpy(), want)
    assert s.t[3] == 0 and s.t[5] == 0 and not top[[3, 5]].any()
    assert bool(torch.isnan(s.t.cpu()[~np.isfinite(top)]).all())


@pytest.mark.parametrize("value", [float("inf"), -float("inf"), float("nan")])
@pytest.mark.parametrize("d", [7, 256, 1021, 2048, 4104])
def test_norm_codes_of_zeros_under_a_weight_that_is_not_finite(cuda, d, value):
    # 0 inf is no number, in a row of zeros too
    x = extreme_rows(d, 1)
    w = torch.ones(d, dtype=torch.bfloat16)
    w[d // 3] = value
    q, s, _, _ = ops.rms_norm_int8(x.to(cuda), w.to(cuda))
    assert bool(torch.isnan(s).all()) and not q.any()

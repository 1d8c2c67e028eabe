"""Forms of the 8-bit products and weight gradients that only some sizes take:
each test names the form (int8_routes) and fails where its sizes no longer
reach it.

Tolerances as in test_gpu_int8_ops.py: the rounding of the result (2^-8) and
T (weight gradient) or 4 (product) times 2^-24 of the magnitudes.  T 2^-24
bounds any order of the sum and is wide for long ones, so each tile's sampled
elements are also held to a relative L2 error of 3e-3: the rounding of the
result is 1.7e-3 and the sum's own error, which walks at random, below 1e-4;
a step left out of a few hundred would be 5e-2.
"""
import ctypes

import numpy as np
import pytest
import torch

from paper_2405_13226_amd import _lib, block_ops as ops

import int8_routes as routes
from parity import log
from test_gpu_int8_ops import B, U, Guarded, at, random_codes

pytestmark = pytest.mark.gpu


def gradient(T, N, seed, dev):
    gen = torch.Generator(device=dev).manual_seed(seed)
    return torch.randn((T, N), generator=gen, device=dev).to(torch.bfloat16)


def check_gradient(q, s, dy, dw, edge):
    """dw against float64 on the first, the last and two other rows of every
    row of tiles, at every column."""
    T, M = q.shape
    rng = np.random.default_rng(T + M)
    rows = np.unique(np.concatenate(
        [np.r_[m, min(m + edge, M) - 1, rng.integers(m, min(m + edge, M), 2)]
         for m in range(0, M, edge)]))
    rows_d = torch.from_numpy(rows).to(q.device)
    x = (q[:, rows_d].float() * s[:, None]).to(torch.bfloat16).double().t().contiguous()
    ref, mag = x @ dy.double(), x.abs() @ dy.double().abs()
    got = dw[rows_d].double()
    assert bool(got.isfinite().all())
    off = (got - ref).abs() - (B * ref.abs() + T * U * mag)
    assert float(off.max()) <= 0, (float(off.max()), int((off > 0).sum()))
    for m in range(0, M, edge):
        mine = torch.from_numpy((rows >= m) & (rows < m + edge)).to(q.device)
        for n in range(0, dy.shape[1], edge):
            g, r = got[mine, n:n + edge], ref[mine, n:n + edge]
            # a few numbers at a matrix's edge have no average rounding
            if r.numel() >= 128:
                assert float((g - r).norm() / r.norm()) <= 3e-3, (m, n)


# The first steps of shared tiles by equal parts, the rest of all of them in
# pieces that workgroups take one after the other.
@pytest.mark.parametrize("T,M,N,n,edge,heads,whole", [
    (4710, 2736, 5944, 1, 256, 1, True), (20012, 4272, 5832, 1, 256, 1, True),
    (16384, 1024, 2816, 2, 256, 2, False), (11504, 320, 3592, 1, 128, 2, False)])
def test_weight_gradients_with_the_rest_in_pieces(cuda, T, M, N, n, edge, heads, whole):
    log(f"wgrad pieces T={T} M={M} N={N} n={n}")
    form = routes.wgrad(T, M, N, n)
    assert form["tails"] > 0 and form["rest"] > 0, form
    assert (form["edge"], form["heads"], form["whole"] > 0) == (edge, heads, whole), form
    q, s = random_codes(T, M, T + M, cuda)
    dys = [gradient(T, N, N + i, cuda) for i in range(n)]
    dw = torch.empty((M, n * N), dtype=torch.bfloat16, device=cuda)
    columns = [dw[:, i * N:(i + 1) * N] for i in range(n)]
    ops.gemm_int8_wgrad_group(q, s, dys, outs=columns)
    for dy, c in zip(dys, columns):
        check_gradient(q, s, dy, c, edge)
    again = ops.gemm_int8_wgrad_group(q, s, dys)
    for a, c in zip(again, columns):
        assert torch.equal(a, c)


def test_weight_gradient_in_pieces_stays_inside_its_buffers(cuda):
    T, M, N = 11504, 320, 3592
    assert routes.wgrad(T, M, N)["tails"] > 0
    lib, st = _lib.lib(), ctypes.c_void_p(torch.cuda.current_stream().cuda_stream)
    q, s = random_codes(T, M, 1, cuda)
    dy = gradient(T, N, 2, cuda)
    need = lib.dd_gemm_i8_wgrad_workspace_bytes(T, M, N, 1)
    dw, ws = Guarded((M, N), torch.bfloat16, cuda), Guarded((need,), torch.uint8, cuda)
    ptrs = lambda t: (ctypes.c_void_p * 1)(t.data_ptr())
    assert lib.dd_gemm_i8_wgrad(at(q), M, at(s), ptrs(dy), N, ptrs(dw.t), N, 1, T, M, N, ws.p,
                                need, st) == 0
    torch.cuda.synchronize()
    assert ws.intact() and dw.intact()
    assert torch.equal(dw.t, ops.gemm_int8_wgrad(q, s, dy))


# T of at most 64 tokens in 256 x 256 tiles: one step, without the loop; then
# two, which is the loop's start and end alone.
@pytest.mark.parametrize("T,M,N,n,steps", [
    (1, 3584, 1792, 1, 1), (45, 3584, 1792, 1, 1), (64, 2032, 2200, 1, 1), (1, 2032, 2200, 1, 1),
    (50, 2048, 2048, 3, 1), (64, 1280, 1280, 3, 1), (65, 2032, 2200, 1, 2),
    (100, 3584, 1792, 1, 2), (128, 2032, 2200, 1, 2)])
def test_weight_gradients_of_one_and_two_steps_in_large_tiles(cuda, T, M, N, n, steps):
    log(f"wgrad large tiles T={T} M={M} N={N} n={n}")
    form = routes.wgrad(T, M, N, n)
    assert form["edge"] == 256 and form["steps"] == steps, form
    # what lies behind the last token is not read into the sums
    q, s = random_codes(T + 40, M, T + M, cuda)
    dys = [gradient(T + 40, N, N + i, cuda) for i in range(n)]
    for dy in dys:
        dy[T:] = float("nan")
    s[T:] = float("inf")
    q, s, dys = q[:T], s[:T], [dy[:T] for dy in dys]
    for dy, dw in zip(dys, ops.gemm_int8_wgrad_group(q, s, dys)):
        check_gradient(q, s, dy, dw, 256)


def check_product(q, s, p, t, r, c):
    """c against float64, every element (the sums of codes are exact in it)."""
    ref = (q.double() @ p.double().t()) * torch.outer(s.double(), t.double())
    mag = ref.abs()
    if r is not None:
        ref, mag = ref + r.double(), mag + r.double().abs()
    off = (c.double() - ref).abs() - (B * ref.abs() + 4 * U * mag)
    assert bool(c.isfinite().all()) and float(off.max()) <= 0, float(off.max())


# Few tokens and more than 16,384 channels: 32 of them a workgroup, two blocks
# of 16; one, two and four blocks of tokens.
@pytest.mark.parametrize("residual", [False, True])
@pytest.mark.parametrize("M,N,K", [
    (M, N, K) for M in (1, 17, 33, 64) for N in (16385, 20001) for K in (16, 1040, 2048)
    if (M, N, K) not in ((33, 20001, 2048), (64, 16385, 2048), (64, 20001, 1040),
                         (64, 20001, 2048))])  # which go to tiles
def test_few_tokens_with_many_channels(cuda, M, N, K, residual):
    log(f"gemm_int8 few M={M} N={N} K={K} residual={residual}")
    assert routes.product(M, N, K) == "few" and N > 16384
    q, s = random_codes(M, K, M + K, cuda, full=True)
    p, t = random_codes(N, K, N + K + 1, cuda, full=True)
    r = gradient(M, N, 9, cuda) if residual else None
    out = Guarded((M, N), torch.bfloat16, cuda)
    ops.gemm_int8(q, s, p, t, residual=r, out=out.t)
    torch.cuda.synchronize()
    assert out.intact()
    check_product(q, s, p, t, r, out.t)


# The large tiles with the residual in the output itself, rows of any
# alignment, whole and ragged tiles, several tiles a workgroup.
@pytest.mark.parametrize("off", [0, 1, 8])
@pytest.mark.parametrize("M,N,K", [(9000, 6152, 912), (16384, 12288, 144)])
def test_large_tiles_add_to_their_output_in_place(cuda, M, N, K, off):
    log(f"gemm_int8 in place M={M} N={N} K={K} off={off}")
    assert routes.product(M, N, K) == "large"
    q, s = random_codes(M, K, 1, cuda)
    p, t = random_codes(N, K, 2, cuda)
    r = gradient(M, N, 3, cuda)
    want = ops.gemm_int8(q, s, p, t, residual=r)
    wide = torch.full((M + 2, N + 24), 5.0, dtype=torch.bfloat16, device=cuda)
    into = wide[1:-1, off:off + N]
    into.copy_(r)
    ops.gemm_int8(q, s, p, t, residual=into, out=into)
    assert torch.equal(into, want)
    keep = torch.ones_like(wide, dtype=torch.bool)
    keep[1:-1, off:off + N] = False
    assert bool((wide[keep] == 5.0).all())
    check_product(q[:512], s[:512], p, t, r[:512], into[:512])
    check_product(q[-300:], s[-300:], p, t, r[-300:], into[-300:])

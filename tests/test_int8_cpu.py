"""The 8-bit operators without a GPU: every refusal of the C ABI (validation
runs on the host before any launch) and of the Python wrappers."""
import ctypes

import numpy as np
import pytest
import torch

from paper_2405_13226_amd import _lib, block_ops as ops

import int8_oracle as O
import int8_routes as routes

OK, NULL, SHAPE, HEADDIM, DOCLENS, WORKSPACE, ALIGN, ALIAS = range(8)


def fake(i, off=0):
    """Addresses 2^30 apart; never read."""
    return ctypes.c_void_p((i + 1) * (1 << 30) + off)


@pytest.fixture(scope="module")
def lib():
    return _lib.lib()


def call(lib, fn, defaults, **kw):
    a = dict(defaults)
    assert set(kw) <= set(a), kw
    a.update(kw)
    return getattr(lib, fn)(*a.values(), None)


NORM = dict(X=fake(0), ldx=512, R=fake(1), ldr=512, w=fake(2), H=fake(3), Y=fake(4),
            rstd=fake(5), rows=8, d=512, eps=1e-5)
NORM8 = dict(X=fake(0), ldx=512, R=fake(1), ldr=512, w=fake(2), H=fake(3), Q=fake(4), ldq=512,
             scales=fake(6), rstd=fake(5), rows=8, d=512, eps=1e-5)


@pytest.mark.parametrize("fn,base", [("dd_rmsnorm_fwd", NORM), ("dd_rmsnorm_int8_fwd", NORM8)])
def test_norm_refusals(lib, fn, base):
    for n in ("X", "w", "H", "R", "rstd") + (("Y",) if "Y" in base else ("Q", "scales")):
        assert call(lib, fn, base, **{n: None}) == NULL, n
    for kw in (dict(rows=0), dict(d=0), dict(d=16385, ldx=1 << 15, ldr=1 << 15), dict(ldx=511),
               dict(ldr=511), dict(eps=0.0), dict(eps=-1.0), dict(eps=float("nan")),
               dict(eps=float("inf")), dict(rows=(1 << 31) - 1, d=1024, ldx=1024, ldr=1024)):
        assert call(lib, fn, base, **kw) == SHAPE, kw
    assert call(lib, fn, base, X=fake(0, 1)) == ALIGN
    assert call(lib, fn, base, rstd=fake(5, 2)) == ALIGN
    out = "Y" if "Y" in base else "Q"
    assert call(lib, fn, base, **{out: fake(0, 64)}) == ALIAS
    assert call(lib, fn, base, H=fake(1)) == ALIAS
    assert call(lib, fn, base, H=fake(4)) == ALIAS
    if fn == "dd_rmsnorm_int8_fwd":
        assert call(lib, fn, base, ldq=500) == SHAPE
        assert call(lib, fn, base, scales=fake(6, 1)) == ALIGN
        assert call(lib, fn, base, scales=fake(5)) == ALIAS


def test_norm_backward_refusals(lib):
    need = lib.dd_rmsnorm_bwd_workspace_bytes(8, 512)
    assert need > 0 and lib.dd_rmsnorm_bwd_workspace_bytes(0, 512) == 0
    assert lib.dd_rmsnorm_bwd_workspace_bytes(8, 16385) == 0
    base = dict(H=fake(0), w=fake(1), rstd=fake(2), dY=fake(3), dRes=fake(4), dX=fake(5),
                dw=fake(6), rows=8, d=512, ws=fake(7), bytes=need)
    for n in ("H", "w", "rstd", "dY", "dX", "dw"):
        assert call(lib, "dd_rmsnorm_bwd", base, **{n: None}) == NULL, n
    assert call(lib, "dd_rmsnorm_bwd", base, rows=0) == SHAPE
    assert call(lib, "dd_rmsnorm_bwd", base, d=20000) == SHAPE
    assert call(lib, "dd_rmsnorm_bwd", base, ws=None) == WORKSPACE
    assert call(lib, "dd_rmsnorm_bwd", base, bytes=need - 1) == WORKSPACE
    assert call(lib, "dd_rmsnorm_bwd", base, ws=fake(7, 2)) == ALIGN
    assert call(lib, "dd_rmsnorm_bwd", base, dX=fake(3)) == ALIAS
    assert call(lib, "dd_rmsnorm_bwd", base, dX=fake(4, 16)) == ALIAS
    assert call(lib, "dd_rmsnorm_bwd", base, ws=fake(6, 16)) == ALIAS


def test_codes_refusals(lib):
    q = dict(X=fake(0), ldx=512, Q=fake(1), ldq=512, scales=fake(2), rows=8, d=512)
    for n in ("X", "Q", "scales"):
        assert call(lib, "dd_quantize", q, **{n: None}) == NULL
    for kw in (dict(rows=0), dict(d=0), dict(d=16385), dict(ldx=500), dict(ldq=500)):
        assert call(lib, "dd_quantize", q, **kw) == SHAPE, kw
    assert call(lib, "dd_quantize", q, X=fake(0, 1)) == ALIGN
    assert call(lib, "dd_quantize", q, Q=fake(0, 512)) == ALIAS
    d = dict(Q=fake(0), ldq=512, scales=fake(1), Y=fake(2), ldy=512, rows=8, d=512)
    for n in ("Q", "scales", "Y"):
        assert call(lib, "dd_dequantize", d, **{n: None}) == NULL
    for kw in (dict(rows=0), dict(d=16385), dict(ldy=500), dict(ldq=500)):
        assert call(lib, "dd_dequantize", d, **kw) == SHAPE, kw
    assert call(lib, "dd_dequantize", d, Y=fake(0, 512)) == ALIAS
    assert call(lib, "dd_dequantize", d, Y=fake(2, 1)) == ALIGN


def test_product_refusals(lib):
    g = dict(A=fake(0), lda=128, sa=fake(1), B=fake(2), ldb=128, sb=fake(3), R=None, C=fake(4),
             ldc=96, M=64, N=96, K=128)
    for n in ("A", "sa", "B", "sb", "C"):
        assert call(lib, "dd_gemm_i8", g, **{n: None}) == NULL, n
    for kw in (dict(M=0), dict(N=0), dict(K=0), dict(K=8), dict(K=120), dict(lda=112),
               dict(ldb=112), dict(ldc=95), dict(K=1 << 17, lda=1 << 17, ldb=1 << 17),
               dict(lda=1 << 23), dict(ldb=1 << 23), dict(M=1 << 20, N=1 << 20, ldc=1 << 20)):
        assert call(lib, "dd_gemm_i8", g, **kw) == SHAPE, kw
    for kw in (dict(lda=136), dict(ldb=136), dict(A=fake(0, 8)), dict(B=fake(2, 4)),
               dict(sa=fake(1, 2)), dict(C=fake(4, 1)), dict(R=fake(5, 1))):
        assert call(lib, "dd_gemm_i8", g, **kw) == ALIGN, kw
    for kw in (dict(C=fake(0, 64)), dict(C=fake(2)), dict(C=fake(1)), dict(C=fake(3, 128)),
               dict(R=fake(4, 2))):
        assert call(lib, "dd_gemm_i8", g, **kw) == ALIAS, kw


def pointers(*ps):
    return (ctypes.c_void_p * len(ps))(*(p.value if p is not None else None for p in ps))


def test_weight_gradient_refusals(lib):
    sizes = lib.dd_gemm_i8_wgrad_workspace_bytes
    need = sizes(64, 96, 128, 2)
    assert need > 64 * 96 * 2
    for bad in ((0, 96, 128, 1), (1 << 25, 96, 128, 1), (64, 92, 128, 1), (64, 96, 124, 1),
                (64, 96, 128, 0), (64, 96, 128, 4)):
        assert sizes(*bad) == 0, bad
    g = dict(Q=fake(0), ldq=96, scales=fake(1), dY=pointers(fake(2), fake(3)), ldy=128,
             dW=pointers(fake(4), fake(5)), ldw=128, n=2, T=64, M=96, N=128, ws=fake(6),
             bytes=need)
    for n in ("Q", "scales", "dY", "dW"):
        assert call(lib, "dd_gemm_i8_wgrad", g, **{n: None}) == NULL, n
    assert call(lib, "dd_gemm_i8_wgrad", g, dY=pointers(fake(2), None)) == NULL
    assert call(lib, "dd_gemm_i8_wgrad", g, dW=pointers(None, fake(5))) == NULL
    for kw in (dict(T=0), dict(T=1 << 25), dict(M=0), dict(M=92), dict(N=100), dict(n=0),
               dict(n=4), dict(ldq=88), dict(ldy=120), dict(ldw=120), dict(ldq=1 << 23),
               dict(ldy=1 << 23)):
        assert call(lib, "dd_gemm_i8_wgrad", g, **kw) == SHAPE, kw
    for kw in (dict(ldq=100), dict(ldy=132), dict(ldw=132), dict(Q=fake(0, 4)),
               dict(dY=pointers(fake(2, 8), fake(3))), dict(dW=pointers(fake(4), fake(5, 8))),
               dict(scales=fake(1, 1)), dict(ws=fake(6, 8))):
        assert call(lib, "dd_gemm_i8_wgrad", g, **kw) == ALIGN, kw
    for kw in (dict(bytes=need - 1), dict(ws=None)):
        assert call(lib, "dd_gemm_i8_wgrad", g, **kw) == WORKSPACE, kw
    for kw in (dict(dW=pointers(fake(4), fake(0))), dict(dW=pointers(fake(1, 64), fake(5))),
               dict(dW=pointers(fake(4), fake(2, 16))), dict(dW=pointers(fake(4), fake(4, 32))),
               dict(ws=fake(0, 16)), dict(ws=fake(3, 32)), dict(ws=fake(5, 16)),
               # column slices of one matrix that overlap
               dict(ldw=256, dW=pointers(fake(4), fake(4, 240)))):
        assert call(lib, "dd_gemm_i8_wgrad", g, **kw) == ALIAS, kw


@pytest.mark.parametrize("M, ok", [((1 << 23) - 128, True), ((1 << 23) - 120, False),
                                  ((1 << 23) - 8, False)])
def test_weight_gradient_has_fewer_than_2_16_parts_of_its_rows(lib, M, ok):
    assert (lib.dd_gemm_i8_wgrad_workspace_bytes(1, M, 8, 1) > 0) == ok


def test_wrappers_refuse_what_is_not_on_a_gpu_or_of_another_type():
    x = torch.zeros(4, 32, dtype=torch.bfloat16)
    q, s = torch.zeros(4, 32, dtype=torch.int8), torch.zeros(4)
    w = torch.zeros(32, dtype=torch.bfloat16)
    for f in (lambda: ops.rms_norm(x, w), lambda: ops.rms_norm_int8(x, w),
              lambda: ops.rms_norm(x[0], w), lambda: ops.rms_norm_backward(x, w, s, x),
              lambda: ops.quantize(x), lambda: ops.quantize([1.0]),
              lambda: ops.dequantize(q, s), lambda: ops.dequantize(x, s),
              lambda: ops.gemm_int8(q, s, q, s), lambda: ops.gemm_int8_wgrad(q, s, x),
              lambda: ops.gemm_int8_wgrad_group(q, s, [x, x])):
        with pytest.raises(ValueError):
            f()


def parts_of(plan, wg):
    """The (tile, first step, steps, slot) that a workgroup computes."""
    if wg < plan["whole"]:
        return [(wg, 0, plan["steps"], -1)]
    i, rest, firsts = wg - plan["whole"], plan["rest"], plan["heads"] * plan["shared"]
    if i < firsts:
        j, tile = divmod(i, plan["shared"])
        first = j * plan["head"]
        return [(plan["whole"] + tile, first, min(plan["head"], plan["steps"] - first), i)]
    w = i - firsts
    at, end, out = w * plan["head"], min((w + 1) * plan["head"], plan["shared"] * rest), []
    while at < end:
        tile, skip = divmod(at, rest)
        n = min(rest - skip, end - at)
        out.append((plan["whole"] + tile, plan["steps"] - rest + skip, n,
                    firsts + w * plan["most"] + len(out)))
        at += n
    return out


@pytest.mark.parametrize("n", [1, 2, 3])
@pytest.mark.parametrize("T,M,N", [(65536, 2048, 5632), (3001, 1040, 1416), (65536, 256, 256),
                                   (4096, 1024, 1024), (16384, 1024, 2816), (700, 4352, 4360),
                                   (65536, 4096, 8192), (200000, 264, 520), (9000, 1800, 5000),
                                   (1, 8, 8), (33554368, 8, 8), (65536, 1024, 2816),
                                   (5000, 1100, 2700), (1200, 640, 640), (2100, 300, 300),
                                   (32832, 256, 256), (20000, 136, 200), (65600, 512, 512),
                                   (60047, 8, 8)])
def test_weight_gradient_plans_cover_every_step_once(T, M, N, n):
    p = routes.wgrad(T, M, N, n)
    assert p["tiles"] == p["whole"] + p["shared"] and p["tiles"] % n == 0
    covered, slots = {}, set()
    firsts = p["heads"] * p["shared"]
    for wg in range(p["whole"] + firsts + p["tails"]):
        parts = parts_of(p, wg)
        assert parts and len(parts) <= p["most"]
        assert sum(k for _, _, k, _ in parts) <= max(p["head"], p["steps"])
        for tile, first, k, slot in parts:
            assert k > 0 and first + k <= p["steps"]
            covered.setdefault(tile, []).append((first, k))
            assert slot < 0 or slot not in slots
            slots.add(slot)
            # and where the last launch looks for it
            rest = p["rest"]
            if slot >= firsts:
                w, i = wg - p["whole"] - firsts, tile - p["whole"]
                assert i * rest // p["head"] <= w <= ((i + 1) * rest - 1) // p["head"]
                assert slot == firsts + w * p["most"] + i - w * p["head"] // rest
    assert sorted(covered) == list(range(p["tiles"]))
    for parts in covered.values():
        at = 0
        for first, k in sorted(parts):
            assert first == at
            at += k
        assert at == p["steps"]
    # a shared tile's workgroups are resident together with the others
    assert firsts + p["tails"] <= routes.CUS


def test_oracle_codes_take_ties_to_even():
    z = np.array([[254.0, 1.0, 3.0, -5.0, 0.0], [0.0] * 5, [np.nan, 1.0, 2.0, 3.0, 4.0]])
    q, top = O.codes(z)
    assert q.tolist() == [[127, 0, 2, -2, 0], [0] * 5, [0] * 5]
    assert top[0] == 254.0 and top[1] == 0.0


def test_block_refuses_other_checkpoint_widths():
    from paper_2405_13226_amd.layer import OpenLMBlock
    with pytest.raises(ValueError):
        OpenLMBlock(512, 8, 768, device="cpu", checkpoint_bits=4)
    assert OpenLMBlock(512, 8, 768, device="cpu").checkpoint_bits == 16


@pytest.mark.parametrize("tiles", [1, 3, 255, 256, 257, 2000, 3008, 16896, 66000])
def test_walks_of_large_tiles_hold_no_tile_behind_the_last(tiles):
    # a wave's lanes hold the next 64 tiles of its workgroup's walk
    grid, seen = min(tiles, routes.CUS), []
    for wg in range(grid):
        n = (tiles - wg + grid - 1) // grid
        seen += [routes.walk(wg, i, grid, tiles) for i in range(n)]
        for i in range(n, n + 64):
            assert 0 <= routes.walk(wg, i, grid, tiles) < tiles, (wg, i)
    assert sorted(seen) == list(range(tiles))


def test_block_refuses_a_width_without_codes():
    from paper_2405_13226_amd.layer import OpenLMBlock
    with pytest.raises(ValueError, match="16384"):
        OpenLMBlock(512, 8, 16640, device="meta", checkpoint_bits=8)
    assert OpenLMBlock(512, 8, 16384, device="meta", checkpoint_bits=8).hidden == 16384
    assert OpenLMBlock(512, 8, 16640, device="meta").hidden == 16640


@pytest.mark.parametrize("rows,cols", [((1 << 32) + 8, 1), (1 << 31, 1), (1, 1 << 31),
                                       (2, (1 << 32) + 16)])
def test_wrappers_refuse_sizes_past_31_bits(rows, cols):
    # (they would reach the C ABI without their upper bits)
    from torch._subclasses.fake_tensor import FakeTensorMode
    with FakeTensorMode():
        x = torch.empty((rows, cols), dtype=torch.bfloat16, device="cuda:0")
        q = torch.empty((rows, cols), dtype=torch.int8, device="cuda:0")
        for t, dtype in ((x, torch.bfloat16), (q, torch.int8)):
            with pytest.raises(ValueError, match="2\\^31"):
                ops._dims(t, "x", dtype)
        ok = torch.empty(((1 << 31) - 1, 1), dtype=torch.bfloat16, device="cuda:0")
        assert ops._dims(ok, "x", torch.bfloat16) == ((1 << 31) - 1, 1, 1)

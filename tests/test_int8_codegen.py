"""Code-generation checks of the 8-bit kernels (CPU: hipcc cross-compiles for
gfx950; nothing runs on a GPU).

* No vector registers spilled.
* No wait for vector memory (`vmcnt`) right before a transposed LDS read: it
  would be one for the loads in flight (tests/test_codegen.py).
* The direct loads to LDS go through inline assembly, in which the compiler
  keeps no distance between a scalar register's write by the vector unit and
  its use as an address: five instructions between the two are required, and
  none of the eight before a load may write one of its scalar operands.
* The first refill of a half of LDS comes after a barrier that follows its
  reads (the 256 x 256 kernels).
"""
import re

import pytest

import test_codegen as C

pytestmark = C.pytestmark


@pytest.mark.parametrize("src", ["dd_rms.hip", "dd_gemm_i8.hip", "dd_wgrad_i8.hip"])
def test_kernels_do_not_spill(src):
    res = C.kernel_resources(C.device_asm(src))
    assert res
    assert not {k: v for k, v in res.items() if v[1] != 0}
    # two workgroups' waves of the row kernels share a SIMD
    assert all(v[0] <= 256 for v in res.values())


@pytest.mark.parametrize("prefix", ["_ZN2dd12wgrad_kernelE", "_ZN2dd18wgrad_small_kernelE",
                                    "_ZN2dd14restore_kernelE"])
def test_no_dma_wait_before_transposed_reads(prefix):
    asm = C.device_asm("dd_wgrad_i8.hip")
    (sym,) = C.symbols(asm, prefix)
    lines = C.kernel_body(asm, sym)
    assert any(ln.startswith("ds_read_b64_tr_b16") for ln in lines)
    if "restore" not in prefix:  # which loads to registers
        assert C.waits_before_transposed_reads(lines) == 0


def scalars(line):
    out = set()
    for a, b, c in re.findall(r"\bs\[(\d+):(\d+)\]|\bs(\d+)\b", line):
        out |= set(range(int(a), int(b) + 1)) if a else {int(c)}
    return out


@pytest.mark.parametrize("src, prefix", [
    ("dd_gemm_i8.hip", "_ZN2dd14gemm_i8_kernelE"), ("dd_gemm_i8.hip", "_ZN2dd20gemm_i8_small_kernelE"),
    ("dd_wgrad_i8.hip", "_ZN2dd12wgrad_kernelE"), ("dd_wgrad_i8.hip", "_ZN2dd18wgrad_small_kernelE")])
def test_scalar_operands_of_direct_loads_are_settled(src, prefix):
    asm = C.device_asm(src)
    (sym,) = C.symbols(asm, prefix)
    lines = [ln.split(";")[0].strip() for ln in C.kernel_body(asm, sym)]
    loads = [i for i, ln in enumerate(lines) if "load_lds" in ln or ln.endswith("offen lds")]
    assert len(loads) >= 8
    for i in loads:
        used = scalars(lines[i])
        for ln in lines[max(0, i - 8):i]:
            if ln.startswith("v_"):
                target = ln.split(",")[0]
                assert not scalars(target) & used, (ln, lines[i])


@pytest.mark.parametrize("src, prefix", [("dd_gemm_i8.hip", "_ZN2dd14gemm_i8_kernelE"),
                                         ("dd_wgrad_i8.hip", "_ZN2dd12wgrad_kernelE")])
def test_first_refill_waits_for_the_reads(src, prefix):
    asm = C.device_asm(src)
    (sym,) = C.symbols(asm, prefix)
    lines = C.kernel_body(asm, sym)
    is_load = [("load_lds" in ln or "offen lds" in ln) for ln in lines]
    started = is_load.index(True)
    first = next(i for i in range(started, len(lines)) if lines[i].startswith("ds_read"))
    load = next(i for i in range(first, len(lines)) if is_load[i])
    assert any(a.startswith("s_waitcnt") and "lgkmcnt(0)" in a and b.startswith("s_barrier")
               for a, b in zip(lines[first:load], lines[first + 1:load]))

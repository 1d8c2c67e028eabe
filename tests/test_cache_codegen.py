"""Code-generation checks of the paged cache's and the log probabilities'
kernels (CPU: hipcc cross-compiles for gfx950; nothing runs on a GPU).

* No vector registers spilled, no scratch memory (an array that a register
  index reaches would go there); the registers that the launch shapes rely on.
* The attention's tiles go through inline assembly: no wait for vector memory
  right before a transposed LDS read, and none of the instructions before a
  direct load may write one of its scalar operands from the vector unit
  (tests/test_int8_codegen.py).
"""
import re

import pytest

import test_codegen as C
from test_int8_codegen import scalars

pytestmark = C.pytestmark


@pytest.mark.parametrize("src", ["dd_cache.hip", "dd_cache_attn.hip", "dd_logprobs.hip"])
def test_kernels_do_not_spill(src):
    asm = C.device_asm(src)
    res = C.kernel_resources(asm)
    assert res
    assert not {k: v for k, v in res.items() if v[1] != 0}
    assert set(re.findall(r"\.amdhsa_private_segment_fixed_size (\d+)", asm)) == {"0"}


def kernels(prefix):
    asm = C.device_asm("dd_cache_attn.hip")
    return [(s, C.kernel_body(asm, s)) for s in C.symbols(asm, "_ZN2dd12_GLOBAL__N_1" + prefix)]


def test_registers_of_the_tile_kernels():
    res = C.kernel_resources(C.device_asm("dd_cache_attn.hip"))
    tiles = {k: v[0] for k, v in res.items() if "11tile_kernelILi" in k}
    assert len(tiles) == 2
    for k, v in tiles.items():  # three waves per SIMD at D = 64, two at 128
        assert v <= (168 if "ILi64E" in k else 256)


@pytest.mark.parametrize("prefix", ["11tile_kernelILi", "10few_kernelILi"])
def test_no_dma_wait_before_transposed_reads(prefix):
    for symbol, lines in kernels(prefix):
        assert any(ln.startswith("ds_read_b64_tr_b16") for ln in lines)
        assert C.waits_before_transposed_reads(lines) == 0, symbol


@pytest.mark.parametrize("prefix", ["11tile_kernelILi", "10few_kernelILi", "14weights_kernelILi"])
def test_scalar_operands_of_direct_loads_are_settled(prefix):
    for symbol, lines in kernels(prefix):
        lines = [ln.split(";")[0].strip() for ln in lines]
        loads = [i for i, ln in enumerate(lines) if "load_lds" in ln]
        assert loads, symbol
        for i in loads:
            used = scalars(lines[i])
            for ln in lines[max(0, i - 8):i]:
                if ln.startswith("v_"):
                    assert not scalars(ln.split(",")[0]) & used, (symbol, ln, lines[i])

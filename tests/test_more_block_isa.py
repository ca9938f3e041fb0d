"""Registers of the kernels for few tokens, 8-bit values and the norms' other forms,
read from the gfx950 assembly that the sources compile to (no GPU needed)."""
import re

import pytest

from test_block_isa import _asm, _sizes


@pytest.fixture(scope="module")
def asm():
    return {src: _asm(src) for src in ("k_few.hip", "k_mx8.hip", "k_mx8_gemm.hip", "k_norm8.hip", "k_norm.hip")}


def test_nothing_in_scratch_memory(asm):
    """(but for norms of more than 16384 columns, four groups of 8 a lane)"""
    for src, text in asm.items():
        scratch = _sizes(text, "private_seg_size", "k_")
        most = {n: v for n, v in scratch.items() if v and not re.search(r"k_block_norm\w*ILi1024ELi4E|norm_grad", n)}
        assert scratch and not most, (src, most)


def test_wavefronts_that_the_launches_plan_for_fit(asm):
    """Registers of 512 per SIMD lane: few tokens four wavefronts per SIMD in both
    launches, product tiles two, lean norms of up to 8192 columns all eight, with
    dropout seven."""
    def at_most(src, name, most, pick=lambda n: True):
        v, a = (_sizes(asm[src], w, name) for w in ("num_vgpr", "num_agpr"))
        seen = [n for n in v if pick(n)]
        assert seen, name
        for n in seen:
            assert v[n] + a[n] <= most, (n, v[n], a[n])

    at_most("k_few.hip", "k_few_", 128)
    at_most("k_mx8_gemm.hip", "k_mx8_gemm_tile", 256)
    at_most("k_norm8.hip", "k_block_norm_mx8", 64, lambda n: re.search(r"ILi\d+ELi1ELb1E", n))
    at_most("k_norm.hip", "k_block_norm", 64, lambda n: re.search(r"k_block_normILi\d+ELi1ELb0ELb1E", n))
    at_most("k_norm.hip", "k_block_norm", 72, lambda n: re.search(r"k_block_normILi\d+ELi1ELb1ELb1E", n))


def test_no_packed_fp32(asm):
    for src, text in asm.items():
        assert not re.search(r"\bv_pk_(add|mul|fma)_f32", text), src

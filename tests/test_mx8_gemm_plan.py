"""Which kernel a product of 8-bit activations and 4-bit weights runs on, on the CPU."""
import os

import pytest

from mx8_gemm_kernels import AT_ONCE, CASES, KERNELS, TILE, kernel
from paper_2608_07814_amd import block as lb
from paper_2608_07814_amd import lorex as lx


@pytest.fixture(scope="module", autouse=True)
def library():
    if not os.path.exists(lx.LIB_PATH):
        from paper_2608_07814_amd import build
        build.build()


@pytest.mark.parametrize("name,glu,M,N,K,G", CASES)
def test_sizes_of_the_gpu_tests_run_on_the_kernel_they_are_for(name, glu, M, N, K, G):
    assert kernel(M, N, K, G, glu) == name
    if not glu:
        assert kernel(M, N - 3, K, G, glu) == name  # (columns of any number)


def test_they_cover_every_kernel_and_form():
    seen = {(name, glu, G > 1) for name, glu, _, _, _, G in CASES}
    assert seen == {(k, glu, groups) for k in KERNELS for glu in (False, True) for groups in ((True,) if k == "rows" else (False, True))}
    for name in AT_ONCE:
        own = [c[1:] for c in CASES if c[0] == name]
        steps = {-(-K // 128) for _, _, _, K, _ in own}
        assert any(n % 2 and n > 4 for n in steps) and any(n % 2 == 0 and n > 4 for n in steps), name
        bm, bn = TILE[name]
        for glu in (False, True):
            assert any(g == glu and -(-M // bm) * -(-N // bn) > AT_ONCE[name] for g, M, N, _, _ in own), name


def test_row_kernels_where_the_tiles_cannot_run():
    for _, glu, M, N, K, G in CASES:
        assert kernel(M, N, K, G, glu, rows_only=True) in ("rows", "rows4")


def test_no_size_takes_a_workspace():
    """(the binding does not ask)"""
    L = lb.lib()
    for _, glu, M, N, K, G in CASES:
        for act in range(4):
            if act != lb.ACT_SWIGLU or glu:
                assert L.lx_mx8_gemm_workspace_bytes(M, N, K, G, act) == 0 and not L.lx_last_error()
    for M, N, K, G in ((1, 4096, 14336, 1), (64, 4096, 14336, 1), (1, 256, 14336, 1), (1, 8, 1 << 24, 1), (1 << 20, 1 << 19, 64, 8192), (0, 1, 8, 1)):
        assert L.lx_mx8_gemm_workspace_bytes(M, N, K, G, 0) == 0 and not L.lx_last_error()

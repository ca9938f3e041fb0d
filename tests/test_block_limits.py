"""Sizes next to 2^31 at the entry points around the expert layer, on the CPU. No
call here reaches a kernel launch."""
import os

import pytest

from paper_2608_07814_amd import block as lb
from paper_2608_07814_amd import lorex as lx

FAKE = 0x10000  # a 256-byte-aligned address that is never dereferenced
MOST = (1 << 31) - 256


@pytest.fixture(scope="module")
def L(root):
    if not os.path.exists(lx.LIB_PATH):
        from paper_2608_07814_amd import build
        build.build()
    return lb.lib()


@pytest.mark.parametrize("M,N", [(MOST + 1, 1), ((1 << 31) - 1, 8), (1, MOST + 1), (8, (1 << 31) - 1)])
@pytest.mark.parametrize("G", [1, 4])
def test_products_whose_last_tile_would_pass_2_31_are_refused(L, M, N, G):
    """The kernels count rows and columns in 32 bits, up to a tile of 256 past the
    last."""
    st = L.lx_mx4_gemm(FAKE, FAKE, 16, FAKE, FAKE, FAKE, FAKE if G > 1 else None, G, M, N, 64, FAKE, lx.LX_F32, FAKE, 1 << 62, None)
    assert st == lx.LX_ERR_UNSUPPORTED, L.lx_last_error()
    assert L.lx_mx4_gemm_workspace_bytes(M, N, 64, G) == 0 and L.lx_last_error()


def test_the_largest_sizes_are_taken(L):
    for M, N in ((MOST, 1), (MOST, 8), (1, MOST), (8, MOST)):
        L.lx_mx4_gemm_workspace_bytes(M, N, 64, 1)
        assert not L.lx_last_error()

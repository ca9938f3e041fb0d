"""lx_route_topk_logits's refusals on the CPU. No call here reaches a kernel launch."""
import os

import pytest

from paper_2608_07814_amd import block as lb
from paper_2608_07814_amd import lorex as lx

FAKE = 0x10000  # a 256-byte-aligned address that is never dereferenced
BAD, UNS, SMALL = lx.LX_ERR_INVALID_ARGUMENT, lx.LX_ERR_UNSUPPORTED, lx.LX_ERR_WORKSPACE_TOO_SMALL


@pytest.fixture(scope="module")
def L(root):
    if not os.path.exists(lx.LIB_PATH):
        from paper_2608_07814_amd import build
        build.build()
    return lb.lib()


@pytest.mark.parametrize("call,code", [
    (dict(logits=None), BAD), (dict(logits=FAKE + 8), BAD), (dict(x=None), BAD), (dict(w=FAKE + 8), BAD), (dict(ids=None), BAD),
    (dict(weights=FAKE + 2), BAD), (dict(ws=None), BAD), (dict(ws=FAKE + 64), BAD), (dict(n=16), SMALL), (dict(E=6), UNS), (dict(d=96), UNS),
    (dict(E=516), UNS), (dict(dt=lx.LX_F32), UNS), (dict(k=0), BAD), (dict(k=65), BAD), (dict(T=-1), BAD), (dict(T=1 << 25), UNS),
    (dict(T=0, x=None, logits=None), lx.LX_OK),
])
def test_refusals(L, call, code):
    a = dict(dict(x=FAKE, w=FAKE, dt=lx.LX_BF16, T=40, d=128, E=64, k=4, ids=FAKE, weights=FAKE, logits=FAKE, ws=FAKE, n=1 << 40), **call)
    st = L.lx_route_topk_logits(a["x"], a["w"], a["dt"], a["T"], a["d"], a["E"], a["k"], a["ids"], a["weights"], a["logits"], a["ws"], a["n"], None)
    assert st == code, L.lx_last_error()
    assert bool(L.lx_last_error()) == (code != lx.LX_OK)

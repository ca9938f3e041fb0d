"""Values that an operator around the layer has no business with, and rows that do
not exist, on the GPU."""
import numpy as np
import pytest
import torch

from oracle import block as O
from paper_2608_07814_amd import block as lb
from gpu_util import require_gpu, say

pytestmark = pytest.mark.gpu


def randn(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return lambda *s: torch.randn(*s, device="cuda", generator=g)


@pytest.mark.parametrize("d", [264, 2048, 8200])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_backward_without_pre_norm_does_not_look_at_the_stream(d, dtype):
    """Without w_pre no gradient depends on h_out: what it holds does not change
    them."""
    require_gpu()
    T = 37
    say(f"block_norm_backward without w_pre T={T} d={d} {dtype}")
    r = randn(d)
    h, y, dh_out = r(T, d).to(dtype), r(T, d).to(dtype), r(T, d).to(dtype)
    kw = dict(w_post=(1 + 0.3 * r(d)).bfloat16(), scale=(1 + 0.3 * r(d)).bfloat16(), gate=torch.sigmoid(r(T)))
    ref = lb.block_norm_backward(h, y, None, dh_out, **kw)
    h[3] = float("nan")
    h[5, 7] = float("inf")
    h[20] = 3e38
    got = lb.block_norm_backward(h, y, None, dh_out, **kw)
    for a, b in zip(got, ref):
        assert (a is None) == (b is None)
        assert a is None or torch.equal(a, b) and torch.isfinite(a).all()

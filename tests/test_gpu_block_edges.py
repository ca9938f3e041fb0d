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


@pytest.mark.parametrize("parts", [("gate", "scale", "pre"), ("scale",), ("pre",)])
@pytest.mark.parametrize("d", [264, 2048, 8200])
def test_backward_without_post_norm_keeps_an_infinite_output_to_itself(d, parts):
    """Without w_post neither dh nor dy depends on y; dgate's row and dscale's column
    of an infinite y do, and no other."""
    require_gpu()
    T = 37
    say(f"block_norm_backward without w_post T={T} d={d} {parts}")
    r = randn(d)
    h, y, dx, dh_out = (r(T, d).bfloat16() for _ in range(4))
    kw = dict(w_pre=(1 + 0.3 * r(d)).bfloat16() if "pre" in parts else None, scale=(1 + 0.3 * r(d)).bfloat16() if "scale" in parts else None,
              gate=torch.sigmoid(r(T)) if "gate" in parts else None)
    dx = dx if "pre" in parts else None
    ref = lb.block_norm_backward(h, y, dx, dh_out, **kw)
    y[4, 9], y[30, d - 1] = float("inf"), float("nan")
    got = lb.block_norm_backward(h, y, dx, dh_out, **kw)
    for name in ("dh", "dy", "dw_pre"):
        a, b = getattr(got, name), getattr(ref, name)
        assert a is b is None or torch.equal(a, b), name
    for name, touched in (("dgate", (4, 30)), ("dscale", (9, d - 1))):
        a, b = getattr(got, name), getattr(ref, name)
        if a is not None:
            keep = torch.ones(len(a), dtype=torch.bool, device="cuda")
            keep[list(touched)] = False
            assert torch.equal(a[keep], b[keep]) and not torch.isfinite(a[~keep]).any(), name

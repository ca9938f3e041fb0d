"""Gradients of the block norms' weights over no rows are zeros, whatever the weights hold."""
import pytest
import torch

from paper_2608_07814_amd import block as lb
from gpu_util import require_gpu

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("bad", [float("inf"), float("nan")])
@pytest.mark.parametrize("drop", [None, 0.0, 0.5])
def test_weights_that_are_not_finite(bad, drop):
    require_gpu()
    d = 264
    e = torch.empty(0, d, device="cuda")
    w = {n: torch.full((d,), bad, device="cuda") for n in ("w_pre", "w_post", "scale")}
    if drop is None:
        r = lb.block_norm_backward(e, e, e, e, **w)
    else:
        r = lb.block_norm_dropout_backward(e, e, e, e, drop, torch.tensor([1, 2], device="cuda"), **w)
    assert not r.dw_pre.any() and not r.dw_post.any() and not r.dscale.any()

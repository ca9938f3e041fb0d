"""The layer for a few tokens where its down projections cancel: the hidden activations keep all 24 bits, whatever the
result's type.

The values are chosen so that fp32 holds every step, exactly: silu(32) is 32 (exp(-32) is below half a step of 1), the
up projections are sums of powers of two, and so are the result's."""
import pytest
import torch

from paper_2608_07814_amd import block as lb
from gpu_util import require_gpu, say

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("T", [1, 5, 8, 17, 64])
@pytest.mark.parametrize("f", [32, 1000])
@pytest.mark.parametrize("x", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("out", [torch.float32, torch.bfloat16])
def test_what_is_left_of_hidden_values_that_cancel(T, f, x, out):
    """Two hidden values 32 (1 + 2^-9 + 2^-18) and 32 (1 + 2^-9), of the first and the last column, enter every output
    with 1 and -1: 2^-13 is left."""
    require_gpu()
    say(f"moe_few, cancelling, T={T} f={f} {x} {out}")
    d, E = 96, 3
    gu, dn = torch.zeros(E, 2 * f, d), torch.zeros(E, d, f)
    gu[:, [0, f - 1], 0] = 1.0                                # gates
    gu[:, [f, 2 * f - 1], 1] = gu[:, [f, 2 * f - 1], 32] = 1.0  # up projections
    gu[:, f, 64] = 1.0
    dn[:, :, 0], dn[:, :, f - 1] = 1.0, -1.0
    ex = lb.Mx4Experts(lb.mx4_quantize(gu.cuda()), lb.mx4_quantize(dn.cuda()))
    assert torch.equal(lb.mx4_dequantize(ex.gate_up, torch.float32).cpu(), gu) and torch.equal(lb.mx4_dequantize(ex.down, torch.float32).cpu(), dn)
    v = torch.zeros(T, d)
    v[:, 0], v[:, 1], v[:, 32], v[:, 64] = 32.0, 1.0, 2.0 ** -9, 2.0 ** -18
    ids = torch.arange(T, device="cuda", dtype=torch.int32).view(T, 1) % E
    w = torch.ones(T, 1, device="cuda")
    got = lb.mx4_moe_few(v.cuda().to(x), ids, w, ex, out_dtype=out)
    assert torch.equal(got, torch.full((T, d), 2.0 ** -13, dtype=out, device="cuda")), got[0, :4]

"""Rows picked from activations, and weights, of which an operand reaches 2^32 bytes: where the sizes choose a row kernel
the sums are those of small operands, bit for bit (its addresses have 64 bits)."""
import pytest
import torch

from paper_2608_07814_amd import block as lb
from gpu_util import require_gpu, say

pytestmark = pytest.mark.gpu


def u8(g, *s, lo, hi):
    return torch.randint(lo, hi, s, device="cuda", generator=g, dtype=torch.uint8)


@pytest.mark.parametrize("M,N", [(1, 512), (14, 264)])
@pytest.mark.parametrize("out", [torch.float32, torch.bfloat16, "mx8"])
def test_few_rows_of_many(M, N, out):
    """Few rows on one group share K over four wavefronts, wherever they lie."""
    require_gpu()
    K = 4096
    rows = (1 << 32) // K + 9
    g = torch.Generator(device="cuda")
    g.manual_seed(M)
    say(f"mx8_gemm, {M} of {rows} rows of {K}, {N} columns, {out}")
    a = lb.Mx8(u8(g, 1 << 16, K, lo=0, hi=127).repeat(17, 1)[:rows].contiguous(), u8(g, rows, K // 32, lo=118, hi=123), K)
    b = lb.Mx4(u8(g, N, K // 2, lo=0, hi=256), u8(g, N, K // 32, lo=120, hi=124), K)
    assert a.codes.numel() >= 1 << 32
    pick = torch.randint(0, rows, (M,), device="cuda", generator=g, dtype=torch.int32)
    pick[0] = rows - 1
    got = lb.mx8_gemm(a, b, row_map=pick, out_dtype=out)
    near = lb.Mx8(a.codes[pick.long()], a.scales[pick.long()], K)
    ref = lb.mx8_gemm(near, b, out_dtype=out)
    for x, y in zip(got, ref) if out == "mx8" else [(got, ref)]:
        assert torch.equal(x, y) if torch.is_tensor(x) else x == y


def test_one_row_on_many_weights():
    """A row on 2^32 bytes of weights and more: the first and last columns against a product of these alone."""
    require_gpu()
    K, cols = 8192, 512
    N = (1 << 32) // (K // 2) + 520
    g = torch.Generator(device="cuda")
    g.manual_seed(5)
    say(f"mx8_gemm, one row on {N} x {K}")
    n = N * K // 2
    codes = u8(g, (4 << 20) + 1031, lo=0, hi=256)
    b = lb.Mx4(codes.repeat(-(-n // codes.numel()))[:n].view(N, K // 2), u8(g, N, K // 32, lo=120, hi=124), K)
    a = lb.mx8_quantize(torch.randn(1, K, device="cuda", generator=g))
    got = lb.mx8_gemm(a, b)
    for at in (slice(0, cols), slice(N - cols, N)):
        few = lb.Mx4(b.codes[at].contiguous(), b.scales[at].contiguous(), K)
        A, B = lb.mx8_dequantize(a, torch.float32).double(), lb.mx4_dequantize(few, torch.float32).double()
        ref, mag = A @ B.t(), A.abs() @ B.abs().t()
        assert ((got[:, at].double() - ref).abs() <= 2.0 ** -24 * (K * mag + ref.abs())).all()

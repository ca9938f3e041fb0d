"""Sums of 8-bit activations and 4-bit weights that cancel, with a bf16 result: what is left of large products
is small ones, which have to be there, on every kernel.

Bounds: the products are exact, and a sum of n of them in fp32 is off by at most 2^-24 n of its terms' magnitudes; the
result is rounded by 2^-8 of itself. Terms that are 0 round nothing, so n counts the others."""
import numpy as np
import pytest
import torch

from oracle import block as O
from paper_2608_07814_amd import block as lb
from gpu_util import require_gpu, say

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
# one group and several; few rows (one wavefront's tile) and many (tiles of 64, 128 and 256 rows)
SIZES = [(3, 64, 256, 1), (40, 96, 2048, 1), (700, 2048, 1024, 1), (1024, 2048, 256, 1), (4096, 4096, 256, 1), (64, 48, 512, 16), (3000, 2048, 512, 4)]


def operands(M, N, K, G, residual, seed):
    """Every row: 448 and, but for `residual`, 448 again, then 14 values of 2^-4 ... under one scale, in the 16 columns
    of one instruction's step that begin at a place of the row's own. Every weight row: 6 and -6 there, and values of 0.5
    and 1 else. The large products are 2688 and cancel, each small one is at most 2^-4 1.75."""
    rng = np.random.default_rng(seed)
    Kp = O.padded(K)
    a = np.zeros((M, Kp), np.uint8)
    small = rng.integers(0x18, 0x20, (M, 14))  # 2^-4 .. 1.875 2^-4
    at = rng.integers(0, K // 16, M)
    for m in range(M):
        a[m, 16 * at[m]] = 0x7E
        a[m, 16 * at[m] + 1] = 0 if residual else 0x7E
        a[m, 16 * at[m] + 2:16 * at[m] + 16] = small[m]
    w = rng.integers(1, 3, (G, N, Kp)).astype(np.uint8)
    w[:, :, 0::16], w[:, :, 1::16] = 0x7, 0xF
    w[:, :, K:] = 0
    one = lambda *s: torch.full(s, 127, dtype=torch.uint8, device="cuda")  # noqa: E731
    return (lb.Mx8(torch.from_numpy(a).cuda(), one(M, Kp // 32), K),
            lb.Mx4(torch.from_numpy(w[:, :, 0::2] | w[:, :, 1::2] << 4).cuda(), one(G, N, Kp // 32), K))


@pytest.mark.parametrize("residual", [False, True])
@pytest.mark.parametrize("M,N,K,G", SIZES)
def test_small_products_are_left(M, N, K, G, residual):
    require_gpu()
    say(f"mx8_gemm, cancelling, {M} x {N} x {K} in {G}, residual {residual}")
    a, b = operands(M, N, K, G, residual, M + N)
    off = torch.linspace(0, M, G + 1).int().cuda() if G > 1 else None
    res = torch.full((M, N), -2688.0, device="cuda") if residual else None
    got = lb.mx8_gemm(a, b, offsets=off, residual=res, out_dtype=torch.bfloat16).double()
    A, B = lb.mx8_dequantize(a, torch.float32).double(), lb.mx4_dequantize(b, torch.float32).double()
    ref = torch.cat([A[lo:hi] @ B[g].t() for g, (lo, hi) in enumerate(zip(off.tolist(), off.tolist()[1:]))]) if G > 1 else A @ B[0].t()
    if residual:
        ref = ref - 2688
    # 16 terms, of magnitudes up to 2688, 2688 (the second product or the residual) and 14 2^-4 1.875, and the residual
    tol = 17 * U * (2 * 2688 + 2) + 2.0 ** -8 * ref.abs()
    assert (ref > 0.4).all()
    bad = (got - ref).abs() > tol
    assert not bad.any(), f"{int(bad.sum())} of {bad.numel()} off, the first {got[bad][0]} for {ref[bad][0]}"

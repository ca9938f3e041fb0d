"""Offsets past 32 bits in the 8-bit values, their products and the layer for few
tokens, on the GPU. Parts that lie beyond are compared, bit for bit, with the same
values at the beginning of memory of their own; the product's sums of K <= 4096 values
do not depend on how many rows there are beside them on the row kernel, and the tiles
form a sum in the same order whatever their size."""
import numpy as np
import pytest
import torch

from oracle import block as O
from paper_2608_07814_amd import block as lb
from gpu_util import require_gpu, say

pytestmark = pytest.mark.gpu


def gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def u8(g, *s, hi=256, lo=0):
    return torch.randint(lo, hi, s, device="cuda", generator=g, dtype=torch.uint8)


def weights(g, E, N, K):
    """K a multiple of 128. (The codes repeat every 4 MiB and 1031 bytes: rows differ.)"""
    n = E * N * K // 2
    some = u8(g, (4 << 20) + 1031)
    codes = some.repeat(-(-n // some.numel()))[:n].view(E, N, K // 2)
    return lb.Mx4(codes, u8(g, E, N, K // 32, lo=118, hi=125), K)


def one(q, e):
    return lb.Mx4(q.codes[e:e + 1].clone(), q.scales[e:e + 1].clone(), q.K)


def test_rounding_and_reading_back():
    require_gpu()
    rows, K = (1 << 25) + 5, 128
    x = torch.randn(1 << 20, K, device="cuda", generator=gen(1)).bfloat16().repeat(33, 1)[:rows]
    say(f"mx8 rounding of {x.numel()} values")
    q = lb.mx8_quantize(x)
    assert q.codes.numel() > 1 << 32
    last = lb.mx8_quantize(x[-1000:].clone())
    assert torch.equal(q.codes[-1000:], last.codes) and torch.equal(q.scales[-1000:], last.scales)
    del x
    back = lb.mx8_dequantize(q)
    assert torch.equal(back[-1000:], lb.mx8_dequantize(last))


@pytest.mark.parametrize("M", [3, 40, 700])
def test_activations_whose_codes_pass_32_bits(M):
    """Rows picked from all over 2^32 + 640 bytes of codes."""
    require_gpu()
    rows, K = (1 << 25) + 5, 128
    g = gen(2)
    a = lb.Mx8(u8(g, 1 << 20, K, hi=127).repeat(33, 1)[:rows], u8(g, rows, K // 32, lo=120, hi=124), K)
    b = weights(g, 1, 192, K)
    pick = torch.randint(0, rows, (M,), device="cuda", generator=g, dtype=torch.int32)
    pick[0], pick[M - 1] = rows - 1, 1 << 25
    say(f"mx8_gemm of {M} of {rows} rows")
    got = lb.mx8_gemm(a, b, row_map=pick)
    few = lb.Mx8(a.codes[pick.long()], a.scales[pick.long()], K)
    A, B = (f(q.codes.cpu().numpy(), q.scales.cpu().numpy(), K) for f, q in ((O.dequantize8, few), (O.dequantize, b)))
    ref, mag = A @ B[0].T, np.abs(A) @ np.abs(B[0].T)
    assert (np.abs(got.cpu().double().numpy() - ref) <= 2.0 ** -24 * (K * mag + np.abs(ref))).all()


@pytest.mark.parametrize("per", [1, 300])
def test_weights_whose_codes_pass_32_bits(per):
    """The rows of the first and of the last of 34 groups of 65536 x 4096."""
    require_gpu()
    E, N, K = 34, 1 << 16, 4096
    g = gen(3)
    b = weights(g, E, N, K)
    assert b.codes.numel() > 1 << 32
    x = lb.mx8_quantize(torch.randn(2 * per, K, device="cuda", generator=g))
    off = torch.tensor([0] + [per] * (E - 1) + [2 * per], dtype=torch.int32, device="cuda")
    say(f"mx8_gemm with {b.codes.numel()} bytes of weights, {per} rows a group")
    got = lb.mx8_gemm(x, b, offsets=off)
    two = lb.Mx4(*(torch.cat([t[:1], t[-1:]]) for t in b[:2]), K)
    ref = lb.mx8_gemm(x, two, offsets=off[[0, 1, E]].contiguous())
    assert torch.isfinite(ref).all() and ref[per:].any()
    A, B = lb.mx8_dequantize(x, torch.float32).double(), lb.mx4_dequantize(one(b, E - 1), torch.float32)[0, -512:].double()
    want, mag = A[per:] @ B.t(), A[per:].abs() @ B.abs().t()
    for r in (got, ref):
        assert ((r[per:, -512:].double() - want).abs() <= 2.0 ** -24 * (K * mag + want.abs())).all()
    if per == 1:  # (both on the row kernel)
        assert torch.equal(got, ref)


@pytest.mark.parametrize("out", ["f32", "mx8"])
def test_results_past_32_bits(out):
    """66000 rows of 65600 columns; the first and last rows against a product of these alone."""
    require_gpu()
    M, N, K = 66000, 65600, 128
    g = gen(4)
    a, b = lb.mx8_quantize(torch.randn(M, K, device="cuda", generator=g)), weights(g, 1, N, K)
    say(f"mx8_gemm of {M * N} results, {out}")
    ends = torch.cat([torch.arange(400), torch.arange(M - 400, M)]).cuda()
    few = lb.Mx8(a.codes[ends], a.scales[ends], K)
    if out == "mx8":
        got, ref = lb.mx8_gemm(a, b, out_dtype="mx8"), lb.mx8_gemm(few, b, out_dtype="mx8")
        assert torch.equal(got.codes[ends], ref.codes) and torch.equal(got.scales[ends], ref.scales)
    else:
        got, ref = lb.mx8_gemm(a, b), lb.mx8_gemm(few, b)
        assert torch.equal(got[ends], ref)


def test_few_tokens_on_experts_past_32_bits():
    require_gpu()
    E, d, f = 34, 4096, 1 << 15
    g = gen(5)
    ex = lb.Mx4Experts(weights(g, E, 2 * f, d), weights(g, E, d, f))
    assert ex.gate_up.codes.numel() > 1 << 32
    x, ids = torch.randn(2, d, device="cuda", generator=g).bfloat16(), torch.tensor([[E - 1], [0]], dtype=torch.int32, device="cuda")
    w = torch.rand(2, 1, device="cuda", generator=g)
    say("moe_few on 34 experts of 32768 x 4096")
    got = lb.mx4_moe_few(x, ids, w, ex)
    last = lb.Mx4Experts(*(lb.Mx4(*(torch.cat([t[:1], t[-1:]]) for t in q[:2]), q.K) for q in ex))
    ref = lb.mx4_moe_few(x, (ids > 0).int(), w, last)
    assert torch.isfinite(ref).all() and torch.equal(got, ref)

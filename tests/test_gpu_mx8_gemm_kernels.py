"""Every kernel of the products of 8-bit activations and 4-bit weights, with one group and several, on the GPU against
the definition in 64 bits (of the values that the library reads back).

Bounds: the products are exact, a sum of K of them in fp32 is off by at most 2^-24 K of its terms' magnitudes; the
activations (slopes at most 1.13) pass that on and add, as the bias and the residual do, 2^-24 * 16 (1 + |z|) of their
result; an fp32 output is rounded by 2^-24 of itself. The order of sums does not depend on the result's type, so bf16 and
8-bit results are the rounding of the fp32 one, bit for bit."""
import numpy as np
import pytest
import torch

from paper_2608_07814_amd import block as lb
from gpu_util import require_gpu, say
from mx8_gemm_kernels import CASES, TILE, kernel

pytestmark = pytest.mark.gpu

U = 2.0 ** -24


def gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def activations(rows, K, g):
    """Rows of very different sizes, with outliers and a row of zeros."""
    x = torch.randn(rows, K, device="cuda", generator=g) * torch.exp2(torch.randint(-6, 7, (rows, 1), device="cuda", generator=g).float())
    x[torch.rand(rows, K, device="cuda", generator=g) < 0.02] *= 30
    x[rows // 2] = 0
    return lb.mx8_quantize(x)


def weights(G, N, K, g, spread=2):
    Kp = lb.mx4_padded(K)
    codes = torch.randint(0, 256, (G, N, Kp // 2), device="cuda", generator=g, dtype=torch.uint8)
    scales = torch.randint(121 - spread, 122 + spread, (G, N, Kp // 32), device="cuda", generator=g, dtype=torch.uint8)
    codes[:, :, K // 2:] = 0
    scales[:, :, -(-K // 32):] = 0
    return lb.Mx4(codes, scales, K)


def groups(M, G, bm, seed):
    """Offsets of groups of sizes around the tile's, none and one among them; the last rows belong to none."""
    if G == 1:
        return None, [(0, 0, M)]
    rng = np.random.default_rng(seed)
    rows = M - 3
    some = [0, 1, bm // 2 + 1, bm - 1, bm + 1]
    some = some[:G - 1]
    size = np.array(some if sum(some) < rows // 2 else [0, 1], int)
    cut = np.sort(rng.integers(0, rows - size.sum() + 1, G - len(size) - 1))
    size = np.concatenate([size, np.diff([0, *cut.tolist(), rows - size.sum()])])
    size = rng.permutation(size)
    off = np.concatenate([[0], np.cumsum(size)])
    assert len(off) == G + 1 and off[-1] == rows
    return torch.tensor(off, dtype=torch.int32, device="cuda"), [(g, int(off[g]), int(off[g + 1])) for g in range(G)]


def reference(a, b, M, parts, row_map, bias, act, res):
    """(result, bound) in 64 bits; rows of no group are NaN."""
    A, B = lb.mx8_dequantize(a, torch.float32).double(), lb.mx4_dequantize(b, torch.float32).double()
    if row_map is not None:
        there = (row_map >= 0) & (row_map < A.shape[0])
        A = torch.where(there[:, None], A[row_map.long().clamp(0, A.shape[0] - 1)], 0.0)
    N = B.shape[1]
    z, mag = (torch.full((M, N), float("nan"), dtype=torch.float64, device="cuda") for _ in range(2))
    for g, lo, hi in parts:
        z[lo:hi], mag[lo:hi] = A[lo:hi] @ B[g].t(), A[lo:hi].abs() @ B[g].abs().t()
        if bias is not None:
            z[lo:hi] += bias[g].double()
            mag[lo:hi] += bias[g].double().abs()
    dz = U * a.K * mag
    if act == lb.ACT_SWIGLU:
        (g, u), (dg, du) = z.chunk(2, 1), dz.chunk(2, 1)
        s = g * torch.sigmoid(g)
        r = s * u
        err = 1.13 * dg * u.abs() + s.abs() * du + 1.13 * dg * du + 16 * U * (1 + g.abs()) * r.abs()
    elif act == lb.ACT_NONE:
        r, err = z, dz
    else:
        r = z * torch.sigmoid(z) if act == lb.ACT_SILU else 0.5 * z * torch.special.erfc(-z * 0.5 ** 0.5)
        err = 1.13 * dz + 16 * U * (1 + z.abs()) * r.abs()
    if res is not None:
        r = r + res.double()
        err = err + U * (r.abs() + res.double().abs())
    return r, err + U * r.abs() + 1e-37


def run(a, b, off, row_map, bias, act, res, out, M):
    """The result in memory that held something else."""
    cols = b.codes.shape[1] // (2 if act == lb.ACT_SWIGLU else 1)
    if out == "mx8":
        cp = lb.mx4_padded(cols)
        to = lb.Mx8(torch.full((M, cp), 0xAA, dtype=torch.uint8, device="cuda"), torch.full((M, cp // 32), 0xBB, dtype=torch.uint8, device="cuda"), cols)
    else:
        to = torch.full((M, cols), 77.0, dtype=out, device="cuda")
    assert lb.mx8_gemm(a, b, offsets=off, row_map=row_map, bias=bias, act=act, residual=res, out=to) is to
    return to


def check(name, glu, M, N, K, G, mapped, act, spread=2):
    say(f"mx8_gemm on {name}: {M} x {N} x {K} in {G}, act {act}, map {mapped}")
    assert kernel(M, N, K, G, glu) == name
    g = gen(M + N + act)
    off, parts = groups(M, G, TILE[name][0], N)
    row_map = None
    rows = M
    if mapped:
        rows = M // 3 + 2
        row_map = torch.randint(0, rows, (M,), device="cuda", generator=g, dtype=torch.int32)
        row_map[::37], row_map[5::91] = -1, rows
    a, b = activations(rows, K, g), weights(G, N, K, g, spread)
    cols = N // 2 if glu else N
    bias = torch.randn(G, N, device="cuda", generator=g).to(torch.bfloat16 if mapped else torch.float32)
    res = torch.randn(M, cols, device="cuda", generator=g).to(torch.float32 if mapped else torch.bfloat16)
    got = run(a, b, off, row_map, bias, act, res, torch.float32, M)
    ref, tol = reference(a, b, M, parts, row_map, bias, act, res)
    end = parts[-1][2]
    assert (got[end:] == 77).all()
    bad = ~((got[:end].double() - ref[:end]).abs() <= tol[:end])
    assert not bad.any(), f"{int(bad.sum())} of {bad.numel()} off, rows {bad.any(1).nonzero()[:5, 0].tolist()}, columns {bad.any(0).nonzero()[:5, 0].tolist()}"
    del ref, tol
    assert torch.equal(run(a, b, off, row_map, bias, act, res, torch.float32, M), got)
    rounded = run(a, b, off, row_map, bias, act, res, torch.bfloat16, M)
    assert torch.equal(rounded[:end], got[:end].bfloat16()) and (rounded[end:] == 77).all()
    if cols % 8 == 0:
        codes, want = run(a, b, off, row_map, bias, act, res, "mx8", M), lb.mx8_quantize(got[:end].contiguous())
        assert torch.equal(codes.codes[:end], want.codes) and torch.equal(codes.scales[:end], want.scales)
        assert (codes.codes[end:] == 0xAA).all() and (codes.scales[end:] == 0xBB).all()
    return a, b, off, row_map, bias, res, got


ACTS = {False: (lb.ACT_NONE, lb.ACT_SILU, lb.ACT_GELU), True: (lb.ACT_SWIGLU,)}


@pytest.mark.parametrize("mapped", [False, True])
@pytest.mark.parametrize("name,glu,M,N,K,G", CASES)
def test_every_form(name, glu, M, N, K, G, mapped):
    require_gpu()
    for act in ACTS[glu]:
        check(name, glu, M, N, K, G, mapped, act)


@pytest.mark.parametrize("name,glu,M,N,K,G", [c for c in CASES if not c[1]])
def test_columns_of_any_number(name, glu, M, N, K, G):
    require_gpu()
    check(name, glu, M, N - 3, K, G, False, lb.ACT_SILU)


@pytest.mark.parametrize("name,glu,M,N,K,G", CASES)
def test_wide_scales(name, glu, M, N, K, G):
    """Weights' scales that differ by 2^80: the products are exact, and sums keep what fp32 does."""
    require_gpu()
    check(name, glu, M, N, K, G, False, ACTS[glu][0], spread=40)


@pytest.mark.parametrize("name,glu,M,N,K,G", CASES)
def test_nan_scales_stay_in_their_row_and_column(name, glu, M, N, K, G):
    require_gpu()
    say(f"mx8_gemm on {name}, NaN scales")
    g = gen(N)
    off, parts = groups(M, G, TILE[name][0], N)
    a, b = activations(M, K, g), weights(G, N, K, g)
    act, end = ACTS[glu][0], parts[-1][2]
    row_map = torch.arange(M, dtype=torch.int32, device="cuda")
    group, lo, hi = max(parts, key=lambda p: p[2] - p[1])
    row_map[lo] = -1  # a missing row in the column's group: 0 whatever the weights hold
    ref = run(a, b, off, row_map, None, act, None, torch.float32, M)
    row, col = hi - 1, (N // 2 if glu else N) - 5
    a.scales[row, -(-K // 32) - 1], b.scales[group, col, 1] = 255, 255
    got = run(a, b, off, row_map, None, act, None, torch.float32, M)
    nan = torch.zeros_like(got, dtype=torch.bool)
    nan[row], nan[lo:hi, col], nan[lo] = True, True, False
    assert torch.equal(torch.isnan(got), nan) and torch.equal(got[~nan], ref[~nan]) and not got[lo].any()


@pytest.mark.parametrize("name,glu,M,N,K,G", CASES)
def test_residual_in_place_and_offsets_past_the_rows(name, glu, M, N, K, G):
    require_gpu()
    g = gen(M)
    off, parts = groups(M, G, TILE[name][0], N)
    a, b = activations(M, K, g), weights(G, N, K, g)
    act = ACTS[glu][0]
    h = torch.randn(M, N // 2 if glu else N, device="cuda", generator=g).bfloat16()
    ref, end = lb.mx8_gemm(a, b, offsets=off, act=act, residual=h, out_dtype=torch.bfloat16), parts[-1][2]
    to = h.clone()
    lb.mx8_gemm(a, b, offsets=off, act=act, residual=to, out=to)
    assert torch.equal(to[:end], ref[:end]) and torch.equal(to[end:], h[end:])
    if G > 1:
        wild = off.clone()
        wild[0], wild[-1] = -7, 1 << 30  # clamped to the rows: the last group gets those of none too
        whole = off.clone()
        whole[-1] = M
        assert torch.equal(lb.mx8_gemm(a, b, offsets=wild, act=act), lb.mx8_gemm(a, b, offsets=whole, act=act))

"""Products of 8-bit activations and 4-bit weights on the GPU against the fp64 oracle.

Bounds, fixed before the first run: a sum of K exact products in fp32 is off by at most
2^-24 K of its terms' magnitudes M. Where the result is rounded to bf16 the products of a
group of 16 may lose what lies more than 13 bits below the exponents of the largest of
them: each loses less than 2^-13 of 2^(that sum of exponents), which is at most the
largest product, so the group loses at most 16 * 2^-13 of the sum of its magnitudes
(normal values lose 1e-5 of the result). The activations (slopes at most 1.13) pass
that on; they and the additions add 2^-24 * 16 (1 + |z|) of their result; an output is rounded by
2^-8 (bf16) or 2^-24 of itself. A result in 8 bits is one whose codes differ from the
oracle's only where a value within that bound does."""
import numpy as np
import pytest
import torch
from scipy.special import ndtr

from oracle import block as O
from paper_2608_07814_amd import block as lb
from paper_2608_07814_amd import lorex as lx
from gpu_util import require_gpu, say
from test_gpu_mx8 import near_oracle

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
DT = {"f32": torch.float32, "bf16": torch.bfloat16}
ACTS = {"none": lb.ACT_NONE, "silu": lb.ACT_SILU, "gelu": lb.ACT_GELU, "swiglu": lb.ACT_SWIGLU}


def host(t):
    return t.detach().cpu().double().numpy()


def activations(rows, K, rng, spread=6):
    x = rng.normal(size=(rows, K)) * np.exp2(rng.integers(-spread, spread + 1, size=(rows, 1)))
    x[rng.random((rows, K)) < 0.02] *= 30
    if rows > 4:
        x[4] = 0
    return lb.mx8_quantize(torch.from_numpy(x.astype(np.float32)).cuda())


def weights(G, N, K, rng, spread=2):
    Kp = O.padded(K)
    codes = rng.integers(0, 256, size=(G, N, Kp // 2)).astype(np.uint8)
    scales = rng.integers(121 - spread, 122 + spread, size=(G, N, Kp // 32)).astype(np.uint8)
    codes[:, :, K // 2:] = 0
    scales[:, :, -(-K // 32):] = 0
    return lb.Mx4(torch.from_numpy(codes).cuda(), torch.from_numpy(scales).cuda(), K)


def values8(q):
    return O.dequantize8(q.codes.cpu().numpy(), q.scales.cpu().numpy(), q.K)


def values4(q):
    return O.dequantize(q.codes.cpu().numpy(), q.scales.cpu().numpy(), q.K)


def slope(act, z):
    return 1.13 if act != "none" else 1.0


def apply(act, z):
    with np.errstate(over="ignore"):
        return z / (1 + np.exp(-z)) if act == "silu" else z * ndtr(z) if act == "gelu" else z


def reference(a, b, M, offsets, row_map, bias, act, res, out):
    """(result, bound of the fp32 arithmetic), rows of no group NaN."""
    A, B = values8(a), values4(b)
    B = B if B.ndim == 3 else B[None]
    z, mag = O.gemm(A, B, M, offsets, row_map), O.gemm(np.abs(A), np.abs(B), M, offsets, row_map)
    products = mag.copy()
    if bias is not None:
        off = [0, M] if offsets is None else [int(v) for v in offsets]
        bias = host(bias).reshape(B.shape[0], -1)
        for g in range(B.shape[0]):
            z[off[g]:off[g + 1]] += bias[g]
            mag[off[g]:off[g + 1]] += np.abs(bias[g])
    dz = U * max(a.K, 32) * mag
    if out == "bf16":
        dz = dz + 2.0 ** -9 * products
    if act == "swiglu":
        f = z.shape[1] // 2
        g, u, dg, du = z[:, :f], z[:, f:], dz[:, :f], dz[:, f:]
        s = apply("silu", g)
        r = s * u
        err = 1.13 * dg * np.abs(u) + np.abs(s) * du + 1.13 * dg * du + 16 * U * (1 + np.abs(g)) * np.abs(r)
    else:
        r = apply(act, z)
        err = slope(act, z) * dz + (0 if act == "none" else 16 * U * (1 + np.abs(z)) * np.abs(r))
    if res is not None:
        r = r + host(res)
        err = err + U * (np.abs(r) + np.abs(host(res)))
    return r, err


def check(a, b, M=None, offsets=None, row_map=None, bias=None, act="none", res=None, out="f32"):
    M = a.codes.shape[0] if M is None else M
    N = b.codes.shape[-2]
    cols = N // 2 if act == "swiglu" else N
    kw = dict(bias=bias, act=ACTS[act], residual=res)
    if offsets is not None:
        kw["offsets"] = torch.tensor(offsets, dtype=torch.int32, device="cuda")
    if row_map is not None:
        kw["row_map"] = torch.tensor(row_map, dtype=torch.int32, device="cuda")
    ref, err = reference(a, b, M, offsets, row_map, bias, act, res, out)
    none = np.isnan(ref).all(1)
    if out == "mx8":
        cp = O.padded(cols)
        to = lb.Mx8(torch.full((M, cp), 0xAA, dtype=torch.uint8, device="cuda"), torch.full((M, cp // 32), 0xBB, dtype=torch.uint8, device="cuda"), cols)
        got = lb.mx8_gemm(a, b, out=to, **kw)
        torch.cuda.synchronize()
        assert got is to and (got.codes.cpu().numpy()[none] == 0xAA).all() and (got.scales.cpu().numpy()[none] == 0xBB).all()
        keep = torch.from_numpy(~none).cuda()
        if (~none).any():
            near_oracle(lb.Mx8(got.codes[keep], got.scales[keep], cols), ref[~none], err[~none] + 1e-37)
        return got
    to = torch.full((M, cols), 77.0, dtype=DT[out], device="cuda")
    got = lb.mx8_gemm(a, b, out=to, **kw)
    torch.cuda.synchronize()
    assert got is to and (host(got)[none] == 77).all()
    g, r = host(got)[~none], ref[~none]
    tol = err[~none] + (2.0 ** -8 if out == "bf16" else U) * np.abs(r) + 1e-37
    bad = ~(np.abs(g - r) <= tol)
    assert not bad.any(), f"{bad.sum()} of {bad.size} off, {np.max(np.abs(g - r) / tol):.3g} of the bound"
    return got


@pytest.mark.parametrize("M,N,K", [(5, 64, 2048), (90, 128, 2048), (300, 512, 2048), (700, 2048, 1024)])
def test_normal_values_in_bf16_lose_only_the_rounding(M, N, K):
    """The bound above is far from what normal values lose: next to the rounding of the
    output (2^-9 of a value at most) 1e-4 of the result's mean size is allowed, ten times
    what was measured; a sum formed in bf16 would be off by 1e-3 of it and more."""
    require_gpu()
    rng = np.random.default_rng(M)
    a, b = lb.mx8_quantize(torch.from_numpy(rng.normal(size=(M, K)).astype(np.float32)).cuda()), weights(1, N, K, rng)
    ref = values8(a) @ values4(b)[0].T
    got = host(lb.mx8_gemm(a, b, out_dtype=torch.bfloat16))
    assert np.all(np.abs(got - ref) <= 2.0 ** -8 * np.abs(ref) + 1e-4 * np.sqrt((ref ** 2).mean()))


def split(M, G, rng, tail=0):
    cut = np.sort(rng.integers(0, M - tail + 1, G - 1)) if G > 1 else np.zeros(0, int)
    return [0, *cut.tolist(), M - tail]


ONE = [(1, 64, 128), (1, 8, 8), (3, 40, 136), (16, 2048, 512), (2, 512, 4096), (17, 130, 264), (33, 256, 640), (64, 96, 2048), (100, 520, 384),
       (129, 64, 1032), (300, 200, 128), (257, 1024, 256), (520, 512, 768), (1, 1000, 14336), (1100, 768, 512), (40, 24, 8), (513, 72, 120)]


@pytest.mark.parametrize("M,N,K", ONE)
@pytest.mark.parametrize("act,out", [("none", "f32"), ("swiglu", "mx8"), ("swiglu", "bf16"), ("silu", "bf16"), ("gelu", "mx8")])
def test_one_group(M, N, K, act, out):
    require_gpu()
    if out == "mx8" and (N // 2 if act == "swiglu" else N) % 8:
        N = -(-N // 16) * 16
    say(f"mx8_gemm {M} x {N} x {K} {act} {out}")
    rng = np.random.default_rng(M + N + K)
    r = lambda *s: torch.from_numpy(rng.normal(size=s).astype(np.float32)).cuda()  # noqa: E731
    cols = N // 2 if act == "swiglu" else N
    check(activations(M, K, rng), weights(1, N, K, rng), act=act, out=out)
    check(activations(M, K, rng), weights(1, N, K, rng), bias=r(1, N).to(DT["bf16" if M % 2 else "f32"]), act=act,
          res=r(M, cols).to(DT["f32" if M % 2 else "bf16"]), out=out)


@pytest.mark.parametrize("N", [1, 7, 30, 65, 131, 258])
def test_columns_of_any_number(N):
    require_gpu()
    rng = np.random.default_rng(N)
    for M in (5, 70, 300):
        bias, res = torch.randn(1, N, device="cuda").bfloat16(), torch.randn(M, N, device="cuda")
        for out in DT:
            check(activations(M, 200, rng), weights(1, N, 200, rng), bias=bias, res=res, act="silu", out=out)
        if N % 2 == 0:
            check(activations(M, 200, rng), weights(1, N, 200, rng), bias=bias, act="swiglu", out="bf16")


GROUPS = [(1, 64, 256, 8), (5, 112, 128, 3), (40, 144, 520, 7), (100, 64, 640, 128), (512, 192, 384, 128), (700, 272, 768, 5), (1500, 128, 256, 9),
          (3000, 320, 136, 16), (300, 80, 128, 1000), (64, 48, 2048, 64), (900, 512, 1024, 3)]


@pytest.mark.parametrize("M,N,K,G", GROUPS)
@pytest.mark.parametrize("act,out", [("none", "bf16"), ("swiglu", "mx8"), ("gelu", "f32"), ("none", "mx8")])
def test_groups(M, N, K, G, act, out):
    require_gpu()
    say(f"mx8_gemm groups {M} x {N} x {K} x {G} {act} {out}")
    rng = np.random.default_rng(M + N + K + G)
    rows = max(M // 2, 3)
    row_map = rng.integers(0, rows, M)
    if M > 4:
        row_map[[1, M // 2]] = -1, rows  # no such rows
    cols = N // 2 if act == "swiglu" else N
    bias = torch.randn(G, N, device="cuda")
    check(activations(rows, K, rng), weights(G, N, K, rng), M, split(M, G, rng, tail=M // 10), row_map, bias=bias, act=act,
          res=torch.randn(M, cols, device="cuda").bfloat16() if M % 4 else None, out=out)


def test_groups_without_rows_and_no_rows():
    require_gpu()
    rng = np.random.default_rng(3)
    a, b = activations(40, 128, rng), weights(6, 64, 128, rng)
    check(a, b, 40, [0, 0, 40, 40, 40, 40, 40], out="bf16")
    check(a, b, 40, [0, 0, 0, 0, 0, 0, 0], out="mx8")
    check(a, b, 40, [0, 7, 7, 7, 20, 20, 33], act="swiglu", out="mx8")
    empty = lb.Mx8(a.codes[:0], a.scales[:0], 128)
    one = lb.Mx4(b.codes[0], b.scales[0], 128)
    assert lb.mx8_gemm(empty, one).shape == (0, 64) and lb.mx8_gemm(empty, one, out_dtype="mx8").codes.shape == (0, 128)
    # no rows of A: every entry of the map is out of range
    got = lb.mx8_gemm(empty, one, row_map=torch.zeros(20, dtype=torch.int32, device="cuda"), bias=torch.ones(64, device="cuda"))
    assert torch.equal(got, torch.ones(20, 64, device="cuda"))


def test_offsets_outside_the_rows_are_clamped():
    require_gpu()
    rng = np.random.default_rng(4)
    a, b = activations(90, 256, rng), weights(3, 64, 256, rng)
    off = lambda *v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
    ref = lb.mx8_gemm(a, b, offsets=off(0, 30, 60, 90))
    assert torch.equal(lb.mx8_gemm(a, b, offsets=off(-5, 30, 60, 1 << 30)), ref)


@pytest.mark.parametrize("M,N,K,G", [(3, 200, 4096, 1), (700, 304, 2048, 1), (900, 256, 1024, 12)])
def test_wide_scales(M, N, K, G):
    """Scales that differ by 2^80: sums whose largest terms are exact."""
    require_gpu()
    rng = np.random.default_rng(M)
    check(activations(M, K, rng, spread=30), weights(G, N, K, rng, spread=40), M, split(M, G, rng) if G > 1 else None, out="f32")


@pytest.mark.parametrize("M", [1, 20, 300])
def test_nan_scales_spread_along_their_row_and_column_only(M):
    require_gpu()
    rng = np.random.default_rng(M)
    a, b = activations(M, 512, rng), weights(1, 256, 512, rng)
    ref = lb.mx8_gemm(a, b)
    a.scales[M // 2, 5] = 255
    b.scales[0, 77, 9] = 255
    row_map = torch.arange(M, dtype=torch.int32, device="cuda")
    if M > 1:
        row_map[0] = -1
    got = lb.mx8_gemm(a, b, row_map=row_map)
    nan = torch.zeros_like(got, dtype=torch.bool)
    nan[M // 2], nan[:, 77] = True, True
    if M > 1:
        nan[0], ref[0] = False, 0
    assert torch.equal(torch.isnan(got), nan) and torch.equal(got[~nan], ref[~nan])


def test_residual_in_place():
    require_gpu()
    rng = np.random.default_rng(8)
    for M in (4, 300):
        a, b = activations(M, 256, rng), weights(1, 128, 256, rng)
        h = torch.randn(M, 128, device="cuda").bfloat16()
        ref = lb.mx8_gemm(a, b, residual=h, out_dtype=torch.bfloat16)
        assert torch.equal(lb.mx8_gemm(a, b, residual=h, out=h), ref)


@pytest.mark.parametrize("M,N,K,G,act,out", [(1, 2000, 2048, 1, "silu", "f32"), (64, 256, 1024, 16, "swiglu", "mx8"), (600, 512, 512, 1, "none", "bf16"),
                                              (2000, 512, 512, 6, "swiglu", "mx8"), (50, 208, 8192, 1, "gelu", "f32")])
def test_same_bits_on_every_run_and_in_a_graph(M, N, K, G, act, out):
    require_gpu()
    rng = np.random.default_rng(M + N)
    a, b = activations(M, K, rng), weights(G, N, K, rng)
    off = torch.tensor(split(M, G, rng), dtype=torch.int32, device="cuda") if G > 1 else None
    kw = dict(offsets=off, act=ACTS[act], out_dtype="mx8" if out == "mx8" else DT[out])
    flat = lambda r: r.codes if isinstance(r, lb.Mx8) else r  # noqa: E731
    ref = flat(lb.mx8_gemm(a, b, **kw)).clone()
    for _ in range(3):
        assert torch.equal(flat(lb.mx8_gemm(a, b, **kw)), ref)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        with torch.cuda.graph(graph, stream=side):
            got = lb.mx8_gemm(a, b, **kw)
    torch.cuda.current_stream().wait_stream(side)
    for _ in range(3):
        flat(got).zero_()
        graph.replay()
        assert torch.equal(flat(got), flat(lb.mx8_gemm(a, b, **kw))) and torch.equal(flat(got), ref)


def test_the_next_product_reads_what_the_first_wrote():
    """gate and up with SwiGLU into 8 bits, down with the residual: the values between
    them are the oracle's rounding of what the first product gives in fp32."""
    require_gpu()
    rng = np.random.default_rng(5)
    for M in (3, 40, 700):
        a, gu, dn = activations(M, 512, rng), weights(1, 400, 512, rng), weights(1, 512, 200, rng)
        h = torch.randn(M, 512, device="cuda")
        mid = lb.mx8_gemm(a, gu, act=lb.ACT_SWIGLU, out_dtype="mx8")
        same = lb.mx8_quantize(lb.mx8_gemm(a, gu, act=lb.ACT_SWIGLU))
        assert torch.equal(mid.codes, same.codes) and torch.equal(mid.scales, same.scales)
        check(mid, dn, res=h)


def test_wrapper_refusals():
    require_gpu()
    rng = np.random.default_rng(9)
    a, b = activations(6, 128, rng), weights(2, 64, 128, rng)
    off = torch.tensor([0, 3, 6], dtype=torch.int32, device="cuda")
    z = lambda *s: torch.zeros(*s, device="cuda")  # noqa: E731
    for bad in (dict(bias=z(64)), dict(bias=z(2, 32)), dict(bias=z(2, 64).half()), dict(residual=z(6, 32)), dict(residual=z(6, 64).double()),
                dict(residual=z(64, 6).t()), dict(out=z(6, 32)), dict(out_dtype=torch.float16), dict(bias=torch.zeros(2, 64)),
                dict(out=lb.Mx8(a.codes, a.scales, 128))):
        with pytest.raises(ValueError):
            lb.mx8_gemm(a, b, offsets=off, **bad)
    with pytest.raises(ValueError):
        lb.mx8_gemm(a, weights(1, 64, 256, rng))
    with pytest.raises(ValueError):
        lb.mx8_gemm(a, weights(1, 63, 128, rng), act=lb.ACT_SWIGLU)
    for bad in (dict(), dict(offsets=off, act=7)):  # several groups without offsets; no such activation
        with pytest.raises(lx.LorexError):
            lb.mx8_gemm(a, b, **bad)
    with pytest.raises(lx.LorexError):
        lb.mx8_gemm(a, weights(1, 36, 128, rng), out_dtype="mx8")

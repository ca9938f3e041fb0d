"""Microscaled 4-bit values on the GPU against the fp64 oracle: codes and scales
equal it; products are exact where every fp32 sum is, and within the summation
bound else."""
import numpy as np
import pytest
import torch

from oracle import block as O
from paper_2608_07814_amd import block as lb
from paper_2608_07814_amd import lorex as lx
from gpu_util import require_gpu, say

pytestmark = pytest.mark.gpu

DT = {"f32": torch.float32, "bf16": torch.bfloat16}


def host(t):
    return t.detach().cpu().double().numpy()


# ---------------------------------------------------------------- rounding
def values(rows, K, dtype, seed=0):
    """Rows of very different magnitudes (subnormal scales among them), with
    zeros, outliers, zero blocks and values that lie on midpoints."""
    rng = np.random.default_rng(seed + 7 * rows + K)
    x = rng.normal(size=(rows, K)) * np.exp2(rng.integers(-20, 20, size=(rows, 1)))
    x *= np.where(rng.random((rows, K)) < 0.02, 40.0, 1.0)
    x[rng.random((rows, K)) < 0.05] = 0
    x[rng.random(rows) < 0.1] = 0
    pick = rng.random((rows, K)) < 0.2
    x[pick] = (rng.integers(-28, 29, size=(rows, K)) / 4.0)[pick]
    if rows > 3:
        x[1] *= 2.0 ** -125 / (np.abs(x[1]).max() + 1e-300)
        x[2] = rng.integers(-9, 10, size=K) * 2.0 ** -133
        x[3, :: max(K // 5, 1)] = 1.5e38
    return torch.from_numpy(x.astype(np.float32)).to(DT[dtype])


@pytest.mark.parametrize("rows,K", [(1, 8), (5, 32), (4, 40), (7, 128), (9, 136), (33, 2048), (1, 14336), (301, 264), (64, 768)])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_rounding_equals_oracle(rows, K, dtype):
    require_gpu()
    say(f"mx4_quantize {rows} x {K} {dtype}")
    x = values(rows, K, dtype)
    codes, scales, _ = O.quantize(x.double().numpy())
    Kp = O.padded(K)
    out = lb.Mx4(torch.full((rows, Kp // 2), 0xAA, dtype=torch.uint8, device="cuda"),
                 torch.full((rows, Kp // 32), 0xAA, dtype=torch.uint8, device="cuda"), K)
    q = lb.mx4_quantize(x.cuda(), out=out)
    torch.cuda.synchronize()
    assert np.array_equal(q.scales.cpu().numpy(), scales)
    got = q.codes.cpu().numpy()
    # (a zero's sign does not change what it stands for)
    ref_v, got_v = O.dequantize(codes, scales, Kp), O.dequantize(got, scales, Kp)
    assert np.array_equal(got_v, ref_v)
    for dt in DT.values():
        back = lb.mx4_dequantize(q, dt)
        assert np.array_equal(host(back), ref_v[:, :K])


def test_blocks_with_infinities_and_nan():
    require_gpu()
    x = values(6, 256, "f32")
    x[0, 3], x[4, 40], x[5, 100], x[5, 255] = float("inf"), float("nan"), -float("inf"), float("nan")
    clean = x.clone()
    for r, b in ((0, 0), (4, 1), (5, 3), (5, 7)):
        clean[r, 32 * b:32 * b + 32] = 0
    q, c = lb.mx4_quantize(x.cuda()), lb.mx4_quantize(clean.cuda())
    v, w = host(lb.mx4_dequantize(q)), host(lb.mx4_dequantize(c))
    bad = np.zeros((6, 8), bool)
    for r, b in ((0, 0), (4, 1), (5, 3), (5, 7)):
        bad[r, b] = True
    assert np.array_equal(q.scales.cpu().numpy() == 255, bad)
    wide = np.repeat(bad, 32, 1)
    assert np.isnan(v[wide]).all() and np.array_equal(v[~wide], w[~wide])


def test_every_code_and_scale_reads_back():
    require_gpu()
    codes = np.tile(np.arange(256, dtype=np.uint8), (256, 1)).reshape(256, 256)
    scales = np.repeat(np.arange(256, dtype=np.uint8)[:, None], 16, 1)
    q = lb.Mx4(torch.from_numpy(codes).cuda(), torch.from_numpy(scales).cuda(), 512)
    ref = O.dequantize(codes, scales, 512)
    for dt in DT.values():
        got = host(lb.mx4_dequantize(q, dt))
        # 2^128 and more (codes past 1.5 under the largest scale) is infinite
        with np.errstate(over="ignore"):
            want = torch.from_numpy(ref).to(torch.float32).double().numpy()
        assert np.array_equal(got, want, equal_nan=True)


@pytest.mark.parametrize("rows,K,dtype", [(3, 8, "f32"), (65, 768, "bf16"), (17, 1024, "f32"), (5, 136, "bf16")])
def test_swiglu_rounding(rows, K, dtype):
    """silu(g) u in fp32 is off by at most 2^-24 * 16 (1 + |g|) relatively (an
    exponential of g, a quotient, two products), so codes may differ from the
    oracle's only that near to a midpoint, scales only that near to a power
    of two."""
    require_gpu()
    say(f"mx4 swiglu {rows} x {K} {dtype}")
    rng = np.random.default_rng(rows + K)
    x = torch.from_numpy(rng.normal(size=(rows, 2 * K)).astype(np.float32) * 3).to(DT[dtype])
    q = lb.mx4_quantize(x.cuda(), act=lb.MX4_SWIGLU)
    x = x.double().numpy()
    v = O.silu_mul(x)
    codes, scales, slack = O.quantize(v)
    rel = 2.0 ** -20 * (1 + np.abs(x[:, :K]).max())
    got_s = q.scales.cpu().numpy()
    top = np.zeros((rows, O.padded(K)))
    top[:, :K] = np.abs(v)
    top = top.reshape(rows, -1, 32).max(2)
    frac = np.abs(top / np.exp2(np.round(np.log2(np.maximum(top, 1e-30)))) - 1)
    same = got_s == scales
    assert np.all(same | (frac <= rel)) and same.mean() > 0.99
    mine, ref = O.dequantize(q.codes.cpu().numpy(), got_s, K), O.dequantize(codes, scales, K)
    ok = np.repeat(same, 32, 1)[:, :K]
    assert np.all((mine == ref)[ok] | (slack[ok] <= 8 * rel)) and np.mean(mine[ok] == ref[ok]) > 0.999


def test_rounding_past_32_bits():
    require_gpu()
    K = 8192
    rows = (1 << 31) // K + 3
    x = torch.zeros(rows, K, dtype=torch.bfloat16, device="cuda")
    t = values(3, K, "bf16").cuda()
    x[-3:] = t
    q, r = lb.mx4_quantize(x), lb.mx4_quantize(t)
    assert torch.equal(q.codes[-3:], r.codes) and torch.equal(q.scales[-3:], r.scales) and not q.codes[:3].any()
    back = lb.mx4_dequantize(q, out=x)
    assert torch.equal(back[-3:], lb.mx4_dequantize(r))


# ---------------------------------------------------------------- products
def operand(lead, K, seed, exps=(127, 129)):
    """Random codes under scales 2^0 .. 2^(exps): sums of products of such values
    are multiples of 1/4 below 2^24 / 4 for K up to 4096, hence exact in fp32 in
    any order. The padding is zero."""
    rng = np.random.default_rng(seed)
    Kp = O.padded(K)
    c = rng.integers(0, 256, size=lead + (Kp // 2,)).astype(np.uint8)
    s = rng.integers(exps[0], exps[1], size=lead + (Kp // 32,)).astype(np.uint8)
    c[..., K // 2:] = 0
    s[..., -(-K // 32):] = 0
    return c, s


def dev(c, s, K):
    return lb.Mx4(torch.from_numpy(c).cuda(), torch.from_numpy(s).cuda(), K)


def run(M, N, K, G=1, rows=None, offsets=None, row_map=None, out="f32", seed=0, exps=(127, 129)):
    rows = M if rows is None else rows
    ac, as_ = operand((rows,), K, seed, exps)
    bc, bs = operand((G, N), K, seed + 1, exps)
    o = torch.full((M, N), 777.0, dtype=DT[out], device="cuda")
    t = lambda v: None if v is None else torch.from_numpy(np.ascontiguousarray(v, dtype=np.int32)).cuda()  # noqa: E731
    lb.mx4_gemm(dev(ac, as_, K), dev(bc, bs, K), offsets=t(offsets), row_map=t(row_map), out=o)
    torch.cuda.synchronize()
    a, b = O.dequantize(ac, as_, K), O.dequantize(bc, bs, K)
    return o, a, b, O.gemm(a, b, M, offsets, row_map)


def exact(o, ref):
    ref = np.where(np.isnan(ref), 777.0, ref)  # rows of no group stay as they were
    want = torch.from_numpy(ref).to(torch.float32).to(o.dtype)
    assert torch.equal(o.cpu(), want), f"{(o.cpu() != want).sum().item()} of {want.numel()} differ"


@pytest.mark.parametrize("M,N,K", [(1, 1, 8), (1, 64, 128), (1, 1000, 4096), (2, 77, 136), (7, 128, 2048), (16, 96, 768), (17, 130, 264),
                                   (31, 257, 1024), (33, 64, 640), (48, 200, 512), (64, 1536, 2048), (65, 300, 896), (128, 256, 256),
                                   (129, 255, 384), (200, 513, 1152), (256, 256, 128), (300, 1000, 1000), (515, 770, 1280), (1025, 384, 512),
                                   (1, 14336, 4096), (2049, 129, 128)])
@pytest.mark.parametrize("out", ["f32", "bf16"])
def test_plain_product(M, N, K, out):
    require_gpu()
    say(f"mx4_gemm M={M} N={N} K={K} {out}")
    o, _, _, ref = run(M, N, K, out=out)
    exact(o, ref)


def ragged(M, G, seed):
    """Offsets of G groups of very different sizes, empty ones among them."""
    rng = np.random.default_rng(seed)
    w = rng.random(G) ** 3 * (rng.random(G) < 0.8)
    w[seed % G] += 0.1
    n = rng.multinomial(M, w / w.sum())
    return np.concatenate([[0], np.cumsum(n)])


@pytest.mark.parametrize("M,N,K,G", [(1, 64, 256, 8), (5, 100, 128, 3), (40, 130, 520, 7), (100, 64, 640, 128), (512, 192, 384, 128),
                                     (700, 257, 768, 5), (1500, 128, 256, 9), (3000, 300, 136, 16), (300, 70, 128, 1000), (64, 33, 2048, 64)])
@pytest.mark.parametrize("out", ["f32", "bf16"])
def test_grouped_product(M, N, K, G, out):
    """Rows gathered from fewer rows of A, some map entries out of range (a row of
    zeros), the last rows in no group."""
    require_gpu()
    say(f"mx4_gemm grouped M={M} N={N} K={K} G={G} {out}")
    rng = np.random.default_rng(M + G)
    off = ragged(M - M // 10, G, M)
    rows = max(M // 3, 1)
    rm = rng.integers(0, rows, size=M)
    rm[rng.random(M) < 0.05] = -1
    rm[rng.random(M) < 0.03] = rows
    o, _, _, ref = run(M, N, K, G, rows, off, rm, out)
    exact(o, ref)


@pytest.mark.parametrize("M,N,K,G", [(20, 64, 8192, 1), (64, 130, 6280, 1), (33, 257, 8056, 1), (60, 100, 6408, 3), (90, 67, 12288, 2), (17, 1, 6144, 1)])
@pytest.mark.parametrize("out", ["f32", "bf16"])
def test_product_with_its_sum_in_parts(M, N, K, G, out):
    """Few tiles and a long K: the parts of a sum go through the workspace. Rows of
    no group stay as they are."""
    require_gpu()
    say(f"mx4_gemm in parts M={M} N={N} K={K} G={G} {out}")
    assert lb.lib().lx_mx4_gemm_workspace_bytes(M, N, K, G) >= 2 * M * N * 4
    off = None if G == 1 else ragged(M - 7, G, M) + 3
    o, _, _, ref = run(M, N, K, G, offsets=off, out=out)
    exact(o, ref)


def test_workspace_refusals():
    require_gpu()
    a, b = dev(*operand((20,), 8192, 1), 8192), dev(*operand((1, 64), 8192, 2), 8192)
    for ws, code in ((torch.empty(256, dtype=torch.uint8, device="cuda"), lx.LX_ERR_WORKSPACE_TOO_SMALL),
                     (torch.empty(1 << 20, dtype=torch.uint8, device="cuda")[128:], lx.LX_ERR_INVALID_ARGUMENT)):
        with pytest.raises(lx.LorexError) as e:
            lb.mx4_gemm(a, b, workspace=ws)
        assert e.value.status == code


def test_offsets_outside_the_rows_are_clamped():
    require_gpu()
    off = np.array([-3, 10, 25, 10 ** 6])
    o, a, b, _ = run(40, 96, 256, 3, 40, off)
    exact(o, O.gemm(a, b, 40, [0, 10, 25, 40]))


def test_no_rows_and_groups_without_rows():
    require_gpu()
    o, _, _, _ = run(5, 64, 128, 4, 5, np.zeros(5))
    assert (o == 777).all()
    q = dev(*operand((0,), 128, 1), 128)
    assert lb.mx4_gemm(q, dev(*operand((2, 16), 128, 2), 128), offsets=torch.zeros(3, dtype=torch.int32, device="cuda")).shape == (0, 16)


@pytest.mark.parametrize("M,N,K,G", [(3, 200, 4096, 1), (700, 300, 2048, 1), (900, 256, 1024, 12)])
def test_wide_scales(M, N, K, G):
    """Scales over 40 powers of two: fp32 accumulation, within K 2^-24 of the sum
    of magnitudes (the bound for any order of the K additions)."""
    require_gpu()
    off = None if G == 1 else ragged(M, G, 4)
    o, a, b, ref = run(M, N, K, G, offsets=off, exps=(107, 147))
    mag = O.gemm(np.abs(a), np.abs(b), M, off)
    assert np.all(np.abs(host(o) - ref) <= K * 2.0 ** -24 * mag)


@pytest.mark.parametrize("M", [1, 20, 300])
def test_nan_scale_spreads_along_its_row_and_column_only(M):
    require_gpu()
    K, N = 512, 130
    ac, as_ = operand((M,), K, 3)
    bc, bs = operand((1, N), K, 4)
    clean = lb.mx4_gemm(dev(ac, as_, K), dev(bc, bs, K))
    as_[M - 1, 5] = 255
    bs[0, 77, 15] = 255
    o = lb.mx4_gemm(dev(ac, as_, K), dev(bc, bs, K))
    nan = torch.zeros(M, N, dtype=torch.bool, device="cuda")
    nan[M - 1] = True
    nan[:, 77] = True
    assert torch.equal(o.isnan(), nan) and torch.equal(o[~nan], clean[~nan])


@pytest.mark.parametrize("M,N,K,G", [(1, 2000, 2048, 1), (64, 256, 1024, 16), (600, 512, 512, 1), (2000, 512, 512, 6), (50, 200, 8192, 1)])
def test_same_bits_on_every_run_and_in_a_graph(M, N, K, G):
    require_gpu()
    off = None if G == 1 else torch.from_numpy(ragged(M, G, 2).astype(np.int32)).cuda()
    a = lb.mx4_quantize(torch.randn(M, K, device="cuda"))
    b = lb.mx4_quantize(torch.randn(G, N, K, device="cuda"))
    ref = lb.mx4_gemm(a, b, offsets=off)
    for _ in range(3):
        assert torch.equal(lb.mx4_gemm(a, b, offsets=off), ref)
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(st):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=st):
            o = lb.mx4_gemm(a, b, offsets=off)
    for _ in range(3):
        o.fill_(5)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(o, ref)
    st2 = torch.cuda.Stream()
    got = lb.mx4_gemm(a, b, offsets=off, stream=st2)
    st2.synchronize()
    assert torch.equal(got, ref)


def test_product_offsets_past_32_bits():
    """A weight matrix beyond 2^32 bytes of codes, and an output beyond 2^32 bytes."""
    require_gpu()
    K, G, N = 4096, 3, 900000
    codes = torch.zeros(G, N, K // 2, dtype=torch.uint8, device="cuda")
    scales = torch.full((G, N, K // 32), 127, dtype=torch.uint8, device="cuda")
    bc, bs = operand((1, 64), K, 9)
    codes[2, -64:] = torch.from_numpy(bc[0]).cuda()
    scales[2, -64:] = torch.from_numpy(bs[0]).cuda()
    for M in (2, 1250):
        ac, as_ = operand((M,), K, 8)
        off = torch.tensor([0, 0, 0, M], dtype=torch.int32, device="cuda")
        o = lb.mx4_gemm(dev(ac, as_, K), lb.Mx4(codes, scales, K), offsets=off)
        ref = O.gemm(O.dequantize(ac, as_, K), O.dequantize(bc, bs, K), M)
        assert np.array_equal(host(o[:, -64:]), ref) and not o[-1, :1000].any()
        del o


def test_wrapper_refusals():
    require_gpu()
    a, b = dev(*operand((4,), 128, 1), 128), dev(*operand((2, 16), 128, 2), 128)
    with pytest.raises(lx.LorexError) as e:
        lb.mx4_gemm(a, b)  # two groups without offsets
    assert e.value.status == lx.LX_ERR_INVALID_ARGUMENT
    off = torch.zeros(3, dtype=torch.int32, device="cuda")
    for kw in (dict(offsets=off[:2]), dict(offsets=off.long()), dict(offsets=off.cpu()), dict(offsets=off, out=torch.empty(4, 15, device="cuda")),
               dict(offsets=off, out=torch.empty(4, 16, device="cuda", dtype=torch.float16)),
               dict(offsets=off, row_map=torch.zeros(4, dtype=torch.int64, device="cuda"))):
        with pytest.raises(ValueError):
            lb.mx4_gemm(a, b, **kw)
    with pytest.raises(ValueError):
        lb.mx4_gemm(lb.Mx4(a.codes, a.scales, 120), b, offsets=off)
    with pytest.raises(ValueError):
        lb.mx4_gemm(lb.Mx4(a.codes, a.scales[:, :3], 128), b, offsets=off)
    with pytest.raises(ValueError):
        lb.mx4_quantize(torch.zeros(2, 64, device="cuda", dtype=torch.float16))
    with pytest.raises(ValueError):
        lb.mx4_quantize(torch.zeros(64, 2, device="cuda").t())
    with pytest.raises(lx.LorexError) as e:
        lb.mx4_quantize(torch.zeros(2, 60, device="cuda"))
    assert e.value.status == lx.LX_ERR_UNSUPPORTED

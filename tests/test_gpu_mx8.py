"""Microscaled 8-bit values on the GPU against the fp64 oracle: rounding of stored
values equals it; the norms' output in 8 bits is one of the codes next to the fp64
norm's value.

Bounds, fixed before the first run: those of the norms' fp32 arithmetic (C = 2^-24 *
256 of the magnitudes that are added up) decide how near to a midpoint or to a
scale's border a value has to be for its code or scale to differ from the oracle's."""
import numpy as np
import pytest
import torch

from oracle import block as O
from paper_2608_07814_amd import block as lb
from gpu_util import require_gpu, say

pytestmark = pytest.mark.gpu

C = 256 * 2.0 ** -24
DT = {"f32": torch.float32, "bf16": torch.bfloat16}


def host(t):
    return None if t is None else t.detach().cpu().double().numpy()


def values(rows, K, dtype, seed=0):
    """Rows of very different magnitudes (subnormal scales among them), with zeros,
    outliers, zero blocks, values on midpoints and largest values around 1.75 2^n."""
    rng = np.random.default_rng(seed + 7 * rows + K)
    x = rng.normal(size=(rows, K)) * np.exp2(rng.integers(-20, 20, size=(rows, 1)))
    x *= np.where(rng.random((rows, K)) < 0.02, 40.0, 1.0)
    x[rng.random((rows, K)) < 0.05] = 0
    x[rng.random(rows) < 0.1] = 0
    pick = rng.random((rows, K)) < 0.2
    x[pick] = (rng.integers(-56, 57, size=(rows, K)) / 32.0)[pick]
    if rows > 3:
        x[1] *= 2.0 ** -125 / (np.abs(x[1]).max() + 1e-300)
        x[2] = rng.integers(-9, 10, size=K) * 2.0 ** -133
        x[3, :: max(K // 5, 1)] = 1.5e38
    if rows > 4:
        x[4, ::32] = np.resize([448.0, 450.0, 446.0, 1.75, 1.7578125, -448.0], x[4, ::32].shape)
    return torch.from_numpy(x.astype(np.float32)).to(DT[dtype])


SIZES = [(1, 8), (5, 32), (4, 40), (7, 128), (9, 136), (33, 2048), (1, 14336), (301, 264), (64, 768)]


@pytest.mark.parametrize("rows,K", SIZES)
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_rounding_equals_oracle(rows, K, dtype):
    require_gpu()
    say(f"mx8_quantize {rows} x {K} {dtype}")
    x = values(rows, K, dtype)
    codes, scales, _ = O.quantize8(x.double().numpy())
    Kp = O.padded(K)
    out = lb.Mx8(torch.full((rows, Kp), 0xAA, dtype=torch.uint8, device="cuda"),
                 torch.full((rows, Kp // 32), 0xAA, dtype=torch.uint8, device="cuda"), K)
    q = lb.mx8_quantize(x.cuda(), out=out)
    torch.cuda.synchronize()
    assert np.array_equal(q.scales.cpu().numpy(), scales)
    ref, got = O.dequantize8(codes, scales, Kp), O.dequantize8(q.codes.cpu().numpy(), scales, Kp)
    assert np.array_equal(got, ref)
    assert np.array_equal(host(lb.mx8_dequantize(q, torch.float32)), ref[:, :K])
    want = torch.from_numpy(ref[:, :K]).to(torch.bfloat16).double().numpy()  # (exact from 2^-133 on)
    assert np.array_equal(host(lb.mx8_dequantize(q)), want)


def test_every_code_and_scale_reads_back():
    require_gpu()
    codes = np.tile(np.arange(256, dtype=np.uint8), (256, 1))
    scales = np.repeat(np.arange(256, dtype=np.uint8)[:, None], 8, 1)
    q = lb.Mx8(torch.from_numpy(codes).cuda(), torch.from_numpy(scales).cuda(), 256)
    ref = O.dequantize8(codes, scales, 256)
    for dt in DT.values():
        with np.errstate(over="ignore"):
            want = torch.from_numpy(ref).to(dt).double().numpy()
        assert np.array_equal(host(lb.mx8_dequantize(q, dt)), want, equal_nan=True)


def test_blocks_with_infinities_and_nan():
    require_gpu()
    x = values(6, 256, "f32")
    clean = x.clone()
    for r, c, v in ((0, 3, np.inf), (4, 40, np.nan), (5, 100, -np.inf), (5, 255, np.nan)):
        x[r, c] = float(v)
        clean[r, c // 32 * 32:c // 32 * 32 + 32] = 0
    q, c = lb.mx8_quantize(x.cuda()), lb.mx8_quantize(clean.cuda())
    v, w = host(lb.mx8_dequantize(q)), host(lb.mx8_dequantize(c))
    bad = q.scales.cpu().numpy() == 255
    assert bad.sum() == 4
    wide = np.repeat(bad, 32, 1)
    assert np.isnan(v[wide]).all() and np.array_equal(v[~wide], w[~wide])


def near_oracle(q, ref, err):
    """Codes and scales of q against fp64 values ref [rows][K] that the kernel has
    within err [rows][K] (absolute)."""
    K = ref.shape[1]
    codes, scales, slack = O.quantize8(ref)
    got_s = q.scales.cpu().numpy()
    Kp = O.padded(K)
    wide = lambda v: np.pad(v, ((0, 0), (0, Kp - K))).reshape(v.shape[0], -1, 32)  # noqa: E731
    top, e = np.abs(wide(ref)).max(2), wide(err).max(2)
    m, _ = np.frexp(np.maximum(top, 1e-300))
    same = got_s == scales
    assert np.all(same | (np.abs(m - 0.875) <= 0.875 * e / np.maximum(top, 1e-300))) and np.all(np.abs(got_s.astype(int) - scales) <= 1)
    mine, want = O.dequantize8(q.codes.cpu().numpy(), got_s, K), O.dequantize8(codes, scales, K)
    ok = np.repeat(same, 32, 1)[:, :K]
    # (the smallest step, 2^-10 of a scale, bounds what a distance is relative to)
    unit = np.exp2(scales.astype(float) - 127).repeat(32, 1)[:, :K]
    assert np.all((mine == want)[ok] | (slack * np.maximum(np.abs(ref), unit * 2.0 ** -10) <= err)[ok])
    assert same.mean() > 0.99 and np.mean((mine == want)[ok]) > 0.99
    pad = q.codes.cpu().numpy()[:, K:]
    assert not pad.any()


@pytest.mark.parametrize("rows,K,dtype", [(3, 8, "f32"), (65, 768, "bf16"), (17, 1024, "f32"), (5, 136, "bf16")])
def test_swiglu_rounding(rows, K, dtype):
    """silu(g) u in fp32 is off by at most 2^-24 * 16 (1 + |g|) relatively."""
    require_gpu()
    say(f"mx8 swiglu {rows} x {K} {dtype}")
    rng = np.random.default_rng(rows + K)
    x = torch.from_numpy(rng.normal(size=(rows, 2 * K)).astype(np.float32) * 3).to(DT[dtype])
    q = lb.mx8_quantize(x.cuda(), act=lb.MX4_SWIGLU)
    v = O.silu_mul(x.double().numpy())
    near_oracle(q, v, 2.0 ** -20 * (1 + np.abs(x[:, :K].double().numpy())) * np.abs(v))


def make(T, d, h="bf16", y="bf16", w="bf16", seed=0, parts=("post", "gate", "scale"), rows=None):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed + 1000 * T + d)
    r = lambda *s: torch.randn(*s, device="cuda", generator=g)  # noqa: E731
    p = dict(h=(3 * r(T, d)).to(DT[h]), y=r(rows or T, d).to(DT[y]), w_pre=(1 + 0.3 * r(d)).to(DT[w]))
    p["w_post"] = (1 + 0.3 * r(d)).to(DT[w]) if "post" in parts else None
    p["scale"] = (0.5 + 0.3 * r(d)).to(DT[w]) if "scale" in parts else None
    p["gate"] = torch.sigmoid(r(T)) if "gate" in parts else None
    return p


def check_norm(p, slot_row=None, slot_weights=None, alpha=0.9, eps=1e-5):
    more = {n: p[n] for n in ("w_pre", "w_post", "scale", "gate")}
    h_out, q = lb.block_norm_mx8(p["h"], p["y"], **more, slot_row=slot_row, slot_weights=slot_weights, residual_scale=alpha, eps=eps)
    same_h, _ = lb.block_norm(p["h"], p["y"], **more, slot_row=slot_row, slot_weights=slot_weights, residual_scale=alpha, eps=eps)
    torch.cuda.synchronize()
    assert torch.equal(h_out, same_h)
    y, mag = host(p["y"]), None
    if slot_row is not None:
        y, mag = O.combine(y, slot_row.cpu().numpy(), host(slot_weights))
    _, ref, _, mag_x = O.block_norm(host(p["h"]), y, **{n: host(v) for n, v in more.items()}, residual_scale=float(np.float32(alpha)),
                                    eps=float(np.float32(eps)), y_mag=mag)
    near_oracle(q, ref, C * mag_x)


@pytest.mark.parametrize("T,d", [(1, 8), (3, 40), (5, 512), (7, 520), (2, 1024), (67, 1032), (1, 2048), (130, 2056), (9, 4096),
                                 (3, 4104), (2, 8192), (2, 8200), (1, 16392), (1, 32768)])
def test_norm_sizes(T, d):
    require_gpu()
    say(f"block_norm_mx8 T={T} d={d}")
    check_norm(make(T, d))


@pytest.mark.parametrize("parts", [("post",), ("gate", "scale"), ()])
@pytest.mark.parametrize("h,y,w", [("bf16", "f32", "bf16"), ("f32", "bf16", "f32"), ("f32", "f32", "f32")])
def test_norm_types_and_parts(h, y, w, parts):
    require_gpu()
    say(f"block_norm_mx8 {h} {y} {w} {parts}")
    check_norm(make(11, 1304, h, y, w, parts=parts))


def test_norm_without_a_block():
    require_gpu()
    p = make(21, 776, parts=())
    h_out, q = lb.block_norm_mx8(p["h"], w_pre=p["w_pre"], eps=1e-5)
    assert h_out is p["h"]
    _, ref, _, mag = O.block_norm(host(p["h"]), None, host(p["w_pre"]), eps=float(np.float32(1e-5)))
    near_oracle(q, ref, C * mag)


@pytest.mark.parametrize("T,d,k", [(1, 2048, 8), (5, 264, 3), (33, 4096, 2)])
def test_norm_combines_slots(T, d, k):
    require_gpu()
    say(f"block_norm_mx8 slots T={T} d={d} k={k}")
    p = make(T, d, y="f32", rows=T * k)
    g = torch.Generator(device="cuda")
    g.manual_seed(5)
    row = torch.randint(-1, T * k, (T, k), device="cuda", generator=g, dtype=torch.int32)
    check_norm(p, row, torch.softmax(torch.randn(T, k, device="cuda", generator=g), 1))


def test_norm_rows_of_zeros_and_of_infinities():
    """eps = 0: a row of zeros gives 0 infinities, that is NaN scales, and its padding
    stays 0; other rows are not touched by it."""
    require_gpu()
    p = make(4, 264, "f32", parts=())
    p["h"][1] = 0
    p["h"][2, 5] = float("inf")
    _, q = lb.block_norm_mx8(p["h"], w_pre=p["w_pre"], eps=0.0)
    v = host(lb.mx8_dequantize(q))
    assert np.isnan(v[1]).all() and np.isnan(v[2, :32]).all() and np.isfinite(v[[0, 3]]).all()
    assert not q.codes[:, 264:].any() and not q.scales[:, 9:].any()


def test_gradients_pass_through_the_rounding():
    """The 8-bit norm's gradient is the unrounded norm's: block_norm_backward from the
    gradient of the values, against differences of a fp64 form along random
    directions."""
    require_gpu()
    p = make(6, 264, "f32", "f32", "f32")
    more = {n: p[n] for n in ("w_pre", "w_post", "scale", "gate")}
    h_out, q = lb.block_norm_mx8(p["h"], p["y"], **more, eps=1e-5)
    g = torch.Generator(device="cuda")
    g.manual_seed(3)
    dx = torch.randn(6, 264, device="cuda", generator=g)
    r = lb.block_norm_backward(h_out, p["y"], dx, None, **more, eps=1e-5)
    eps = float(np.float32(1e-5))
    base = {n: host(v) for n, v in more.items()}
    rng = np.random.default_rng(0)
    for name, at, got in (("h", "h", r.dh), ("y", "y", r.dy), ("w_pre", "w_pre", r.dw_pre), ("scale", "scale", r.dscale), ("gate", "gate", r.dgate)):
        v = rng.normal(size=tuple(p[at].shape))
        step = 1e-5

        def loss(s):
            a = {"h": host(p["h"]), "y": host(p["y"]), **base}
            a[name] = a[name] + s * v
            x = O.block_norm(a.pop("h"), a.pop("y"), **a, eps=eps)[1]
            return (x * host(dx)).sum()

        diff = (loss(step) - loss(-step)) / (2 * step)
        # (fp32 rounding of h_out and of the gradients: 2^-24 C's share of the terms' magnitude)
        assert abs(diff - (host(got) * v).sum()) <= 2 * C * np.abs(host(got) * v).sum() + 1e-6, name


def test_norm_in_a_graph_and_in_place():
    require_gpu()
    p = make(9, 1032)
    more = {n: p[n] for n in ("w_pre", "w_post", "scale", "gate")}
    ref_h, ref = lb.block_norm_mx8(p["h"], p["y"], **more)
    h, work = p["h"].clone(), p["h"].clone()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        q = lb.mx8_quantize(work)
        with torch.cuda.graph(graph, stream=side):
            lb.block_norm_mx8(work, p["y"], **more, h_out=work, x=lb.Mx8(q.codes, q.scales, 1032))
    torch.cuda.current_stream().wait_stream(side)
    for _ in range(3):
        work.copy_(h)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(work, ref_h) and torch.equal(q.codes, ref.codes) and torch.equal(q.scales, ref.scales)


def test_empty():
    require_gpu()
    h = torch.empty(0, 64, device="cuda", dtype=torch.bfloat16)
    w = torch.ones(64, device="cuda", dtype=torch.bfloat16)
    h_out, q = lb.block_norm_mx8(h, h, w_pre=w)
    assert h_out.shape == (0, 64) and q.codes.shape == (0, 128) and q.scales.shape == (0, 4)
    assert lb.mx8_quantize(h).codes.shape == (0, 128) and lb.mx8_dequantize(q).shape == (0, 64)


@pytest.mark.parametrize("x", ["bf16", "f32"])
def test_norm_with_its_values_too(x):
    require_gpu()
    for T, d in ((3, 40), (5, 1304), (2, 8200)):
        p = make(T, d)
        more = {n: p[n] for n in ("w_pre", "w_post", "scale", "gate")}
        values = torch.empty(T, d, device="cuda", dtype=DT[x])
        h_out, q = lb.block_norm_mx8(p["h"], p["y"], **more, x_values=values)
        ref_h, ref = lb.block_norm(p["h"], p["y"], **more, x_dtype=DT[x])
        _, only = lb.block_norm_mx8(p["h"], p["y"], **more)
        assert torch.equal(h_out, ref_h) and torch.equal(values, ref)
        assert torch.equal(q.codes, only.codes) and torch.equal(q.scales, only.scales)

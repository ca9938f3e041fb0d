"""Dropout inside the block norms on the GPU against the fp64 oracle.

Bounds, fixed before the first run: those of the norms without it (2^-8 or 2^-24 for
the output's rounding, C = 2^-24 * 256 of the magnitudes that are added up); the
mask is exact, its factor off by 2^-24."""
import numpy as np
import pytest
import torch

from oracle import block as O
from paper_2608_07814_amd import block as lb
from gpu_util import require_gpu, say

pytestmark = pytest.mark.gpu

C = 256 * 2.0 ** -24
DT = {"f32": torch.float32, "bf16": torch.bfloat16}
SEED, OFFSET = 0x1234567890ABCDEF, (7 << 32) + 11


def host(t):
    return None if t is None else t.detach().cpu().double().numpy()


def rng_of(seed=SEED, offset=OFFSET):
    return torch.tensor([seed, offset], dtype=torch.int64, device="cuda")


def within(name, got, ref, mag):
    g, r = host(got), np.asarray(ref)
    unit = 2.0 ** -8 if got.dtype == torch.bfloat16 else 2.0 ** -24
    tol = C * np.asarray(mag) + unit * np.abs(r) + 1e-37
    bad = ~(np.abs(g - r) <= tol)
    assert g.shape == r.shape and not bad.any(), f"{name}: {bad.sum()} of {bad.size} off, {np.max(np.abs(g - r) / tol):.3g} of the bound"


def make(T, d, h="bf16", y="bf16", x="bf16", w="bf16", seed=0, parts=("post", "gate", "scale", "pre")):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed + 1000 * T + d)
    r = lambda *s: torch.randn(*s, device="cuda", generator=g)  # noqa: E731
    p = dict(h=(3 * r(T, d)).to(DT[h]), y=r(T, d).to(DT[y]), dx=r(T, d).to(DT[x]), dh_out=r(T, d).to(DT[h]))
    p["w_pre"] = (1 + 0.3 * r(d)).to(DT[w]) if "pre" in parts else None
    p["w_post"] = (1 + 0.3 * r(d)).to(DT[w]) if "post" in parts else None
    p["scale"] = (0.5 + 0.3 * r(d)).to(DT[w]) if "scale" in parts else None
    p["gate"] = torch.sigmoid(r(T)) if "gate" in parts else None
    return p


def weights(p):
    return {n: p[n] for n in ("w_pre", "w_post", "scale", "gate")}


def check(p, drop, x="bf16", alpha=0.9, eps=1e-5, seed=SEED, offset=OFFSET):
    T, d = p["h"].shape
    rng = rng_of(seed, offset)
    keep = O.dropout_keep(T, d, drop, seed & (1 << 64) - 1, offset & (1 << 64) - 1)
    more = dict(**{n: host(v) for n, v in weights(p).items()}, residual_scale=float(np.float32(alpha)), eps=float(np.float32(eps)), keep=keep)
    h_out, xo = lb.block_norm_dropout(p["h"], p["y"], drop, rng, **weights(p), residual_scale=alpha, eps=eps, x_dtype=DT[x])
    torch.cuda.synchronize()
    ref_h, ref_x, mag_h, mag_x = O.block_norm(host(p["h"]), host(p["y"]), **more)
    within("h_out", h_out, ref_h, mag_h)
    if ref_x is None:
        assert xo is None
    else:
        within("x", xo, ref_x, mag_x)
    # (from a stream after the block of its own: p["h"])
    r = lb.block_norm_dropout_backward(p["h"], p["y"], p["dx"] if p["w_pre"] is not None else None, p["dh_out"], drop, rng, **weights(p),
                                       residual_scale=alpha, eps=eps)
    torch.cuda.synchronize()
    ref = O.block_norm_grads(host(p["h"]), host(p["y"]), host(p["dx"]), host(p["dh_out"]), **more)
    got = {n: v for n, v in r._asdict().items() if v is not None}
    assert set(got) == set(ref)
    for n, (v, mag) in ref.items():
        within(n, got[n], v, mag)


SIZES = [(1, 8), (3, 40), (5, 512), (7, 520), (2, 1024), (67, 1032), (1, 2048), (130, 264), (9, 4096), (3, 4104), (2, 8192), (2, 8200),
         (1, 16392), (1, 32768), (300, 64)]


@pytest.mark.parametrize("T,d", SIZES)
def test_sizes(T, d):
    require_gpu()
    say(f"dropout T={T} d={d}")
    check(make(T, d), 0.1)


@pytest.mark.parametrize("parts", [("post", "gate", "scale", "pre"), ("post", "pre"), ("pre",), ("scale", "gate"), ()])
@pytest.mark.parametrize("h,y,x,w", [("bf16", "f32", "bf16", "bf16"), ("f32", "bf16", "bf16", "f32"), ("f32", "f32", "f32", "f32")])
def test_types_and_parts(h, y, x, w, parts):
    require_gpu()
    say(f"dropout {h} {y} {x} {w} {parts}")
    check(make(13, 1304, h, y, x, w, parts=parts), 0.3, x=x)


@pytest.mark.parametrize("drop", [2.0 ** -16, 0.05, 0.5, 0.9, 1 - 2.0 ** -16])
def test_shares(drop):
    require_gpu()
    check(make(5, 264, "f32", "f32", "f32", "f32"), drop, x="f32")


@pytest.mark.parametrize("seed,offset", [(0, 0), (-1, -1), (-(1 << 63), (1 << 63) - 1), (5, 1 << 32)])
def test_keys(seed, offset):
    require_gpu()
    check(make(4, 40), 0.5, seed=seed, offset=offset)


def test_none_is_the_plain_norm():
    require_gpu()
    p = make(9, 520)
    a, b = lb.block_norm(p["h"], p["y"], **weights(p)), lb.block_norm_dropout(p["h"], p["y"], 0.0, rng_of(), **weights(p))
    assert all(torch.equal(u, v) for u, v in zip(a, b))
    a = lb.block_norm_backward(p["h"], p["y"], p["dx"], p["dh_out"], **weights(p))
    b = lb.block_norm_dropout_backward(p["h"], p["y"], p["dx"], p["dh_out"], 0.0, rng_of(), **weights(p))
    assert all(torch.equal(u, v) for u, v in zip(a, b))


def test_share_and_independence():
    """Kept shares within five deviations of a binomial's, over all values, per bit
    position of the generator's words, and of pairs (neighbours, rows, offsets)."""
    require_gpu()
    T, d, q = 512, 2048, 0.25
    h = torch.zeros(T, d, device="cuda")
    y = torch.ones(T, d, device="cuda")
    draw = lambda o: lb.block_norm_dropout(h, y, q, rng_of(offset=o))[0] > 0  # noqa: E731
    a, b = draw(1), draw(2)

    def near(x, share):
        n = x.numel()
        assert abs(x.float().mean().item() - share) <= 5 * (share * (1 - share) / n) ** 0.5

    near(a, 1 - q)
    for c in range(8):
        near(a[:, c::8], 1 - q)
    for pair in (a[:, :-1] & a[:, 1:], a[:-1] & a[1:], a & b):
        near(pair, (1 - q) ** 2)


def test_dropped_values_are_not_looked_at():
    """Without w_post an infinite or NaN output counts only where it is kept."""
    require_gpu()
    p = make(3, 64, "f32", "f32", "f32", "f32", parts=("scale",))
    keep = O.dropout_keep(3, 64, 0.5, SEED, OFFSET) > 0
    gone = torch.from_numpy(~keep).cuda()
    clean = lb.block_norm_dropout(p["h"], p["y"], 0.5, rng_of(), scale=p["scale"])[0]
    grads = lb.block_norm_dropout_backward(clean, p["y"], None, p["dh_out"], 0.5, rng_of(), scale=p["scale"])
    for v in (float("inf"), float("nan")):
        y = torch.where(gone, torch.full_like(p["y"], v), p["y"])
        assert torch.equal(lb.block_norm_dropout(p["h"], y, 0.5, rng_of(), scale=p["scale"])[0], clean)
        again = lb.block_norm_dropout_backward(clean, y, None, p["dh_out"], 0.5, rng_of(), scale=p["scale"])
        assert torch.equal(again.dscale, grads.dscale) and torch.equal(again.dy, grads.dy) and torch.equal(again.dh, grads.dh)


@pytest.mark.parametrize("case", ["nan", "zeros"])
def test_dropped_values_are_0_where_the_row_has_no_norm(case):
    """With w_post a NaN, or a row of zeros without eps, leaves the row without finite
    normalised values: kept ones are NaN, dropped ones count as 0 all the same."""
    require_gpu()
    p = make(3, 520)
    p["y"][1] = 0
    if case == "nan":
        p["y"][1, 77] = float("nan")
    keep = torch.from_numpy(O.dropout_keep(3, 520, 0.5, SEED, OFFSET) > 0).cuda()
    h_out, _ = lb.block_norm_dropout(p["h"], p["y"], 0.5, rng_of(), w_pre=p["w_pre"], w_post=p["w_post"], gate=p["gate"], eps=0.0)
    assert torch.equal(torch.isnan(h_out[1]), keep[1]) and torch.equal(h_out[1][~keep[1]], p["h"][1][~keep[1]])
    assert torch.isfinite(h_out[[0, 2]]).all()


def test_gradients_against_differences():
    """Along random directions, the mask held fixed by its key."""
    require_gpu()
    p = make(5, 72, "f32", "f32", "f32", "f32")
    keep = O.dropout_keep(5, 72, 0.3, SEED, OFFSET)
    eps = float(np.float32(1e-5))
    base = dict(h=host(p["h"]), y=host(p["y"]), **{n: host(v) for n, v in weights(p).items()})
    h_out, _ = lb.block_norm_dropout(p["h"], p["y"], 0.3, rng_of(), **weights(p), eps=1e-5)
    r = lb.block_norm_dropout_backward(h_out, p["y"], p["dx"], p["dh_out"], 0.3, rng_of(), **weights(p), eps=1e-5)
    gen = np.random.default_rng(1)

    def loss(a):
        a = dict(a)
        o, x = O.block_norm(a.pop("h"), a.pop("y"), **a, eps=eps, keep=keep)[:2]
        return (x * host(p["dx"])).sum() + (o * host(p["dh_out"])).sum()

    for name, got in (("h", r.dh), ("y", r.dy), ("w_pre", r.dw_pre), ("w_post", r.dw_post), ("scale", r.dscale), ("gate", r.dgate)):
        v, step = gen.normal(size=base[name].shape), 1e-5
        diff = (loss({**base, name: base[name] + step * v}) - loss({**base, name: base[name] - step * v})) / (2 * step)
        assert abs(diff - (host(got) * v).sum()) <= 2 * C * np.abs(host(got) * v).sum() + 1e-6, name


def test_graph_draws_anew_when_the_offset_moves_on():
    """Forward and backward captured; the program moves the offset on between the
    replays, and an eager pass on the same leaves lives beside it."""
    require_gpu()
    p = make(33, 520)
    rng = rng_of(offset=100)
    eager = lambda o: lb.block_norm_dropout(p["h"], p["y"], 0.2, rng_of(offset=o), **weights(p))  # noqa: E731
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        with torch.cuda.graph(graph, stream=side):
            h_out, x = lb.block_norm_dropout(p["h"], p["y"], 0.2, rng, **weights(p))
            r = lb.block_norm_dropout_backward(h_out, p["y"], p["dx"], p["dh_out"], 0.2, rng, **weights(p))
    torch.cuda.current_stream().wait_stream(side)
    seen = []
    for i in range(3):
        graph.replay()
        torch.cuda.synchronize()
        ref_h, ref_x = eager(100 + i)
        ref = lb.block_norm_dropout_backward(ref_h, p["y"], p["dx"], p["dh_out"], 0.2, rng_of(offset=100 + i), **weights(p))
        assert torch.equal(h_out, ref_h) and torch.equal(x, ref_x)
        assert all(torch.equal(u, v) for u, v in zip(r, ref))
        seen.append(h_out.clone())
        rng[1] += 1
    assert not torch.equal(seen[0], seen[1])


def test_empty():
    require_gpu()
    p = make(2, 64)
    e = {n: p[n][:0] for n in ("h", "y", "dx", "dh_out")}
    w = dict(weights(p), gate=p["gate"][:0])
    h_out, x = lb.block_norm_dropout(e["h"], e["y"], 0.5, rng_of(), **w)
    assert h_out.shape == x.shape == (0, 64)
    r = lb.block_norm_dropout_backward(e["h"], e["y"], e["dx"], e["dh_out"], 0.5, rng_of(), **w)
    assert not r.dw_pre.any() and not r.dw_post.any() and not r.dscale.any()

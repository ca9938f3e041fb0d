"""Block norms on the GPU against the fp64 oracle.

Bounds, fixed before the first run: an output is rounded once (relative 2^-8
in bf16, 2^-24 in fp32); the fp32 arithmetic before it adds C = 2^-24 * 256 of
the magnitudes that are added up (row sums go through at most 32 serial and 14
tree additions, weight gradients through at most 100 serial ones at these
sizes, and a norm factor is off by half of its sum's error)."""
import numpy as np
import pytest
import torch

from oracle import block as O
from paper_2608_07814_amd import block as lb
from paper_2608_07814_amd import lorex as lx
from gpu_util import require_gpu, say

pytestmark = pytest.mark.gpu

C = 256 * 2.0 ** -24
DT = {"f32": torch.float32, "bf16": torch.bfloat16}


def unit(t):
    return 2.0 ** -8 if t.dtype == torch.bfloat16 else 2.0 ** -24


def host(t):
    return None if t is None else t.detach().cpu().double().numpy()


def within(name, got, ref, mag):
    g, r = host(got), np.asarray(ref)
    assert g.shape == r.shape, name
    tol = C * np.asarray(mag) + unit(got) * np.abs(r) + 1e-37
    bad = ~(np.abs(g - r) <= tol)
    assert not bad.any(), f"{name}: {bad.sum()} of {bad.size} off, worst {np.max(np.abs(g - r) / tol):.3g} of the bound"


def make(T, d, h="bf16", y="bf16", x="bf16", w="bf16", seed=0, k=0, parts=("post", "gate", "scale", "pre"), rows=None):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed + 1000 * T + d)
    r = lambda *s: torch.randn(*s, device="cuda", generator=g)  # noqa: E731
    p = dict(h=(3 * r(T, d)).to(DT[h]), y=r(rows or T, d).to(DT[y]), dx=r(T, d).to(DT[x]), dh_out=r(T, d).to(DT[h]))
    p["w_pre"] = (1 + 0.3 * r(d)).to(DT[w]) if "pre" in parts else None
    p["w_post"] = (1 + 0.3 * r(d)).to(DT[w]) if "post" in parts else None
    p["scale"] = (0.5 + 0.3 * r(d)).to(DT[w]) if "scale" in parts else None
    p["gate"] = torch.sigmoid(r(T)) if "gate" in parts else None
    return p


def weights(p):
    return {n: p[n] for n in ("w_pre", "w_post", "scale", "gate")}


def check_forward(p, x="bf16", alpha=0.9, eps=1e-5, slot_row=None, slot_weights=None):
    h_out, xo = lb.block_norm(p["h"], p["y"], **weights(p), slot_row=slot_row, slot_weights=slot_weights,
                              residual_scale=alpha, eps=eps, x_dtype=DT[x])
    torch.cuda.synchronize()
    alpha, eps = float(np.float32(alpha)), float(np.float32(eps))
    y, mag = host(p["y"]), None
    if slot_row is not None:
        y, mag = O.combine(y, slot_row.cpu().numpy(), host(slot_weights))
    ref_h, ref_x, mag_h, mag_x = O.block_norm(host(p["h"]), y, **{n: host(v) for n, v in weights(p).items()},
                                              residual_scale=alpha, eps=eps, y_mag=mag)
    if p["y"] is None:
        assert h_out is p["h"]
    else:
        within("h_out", h_out, ref_h, mag_h)
    if ref_x is None:
        assert xo is None
    else:
        within("x", xo, ref_x, mag_x)


SIZES = [(1, 8), (3, 40), (5, 512), (7, 520), (2, 1024), (67, 1032), (1, 2048), (130, 2056), (9, 4096), (3, 4104), (2, 8192),
         (2, 8200), (1, 16392), (1, 32768)]
PARTS = [("post", "gate", "scale", "pre"), ("post", "pre"), ("pre",), ("gate",), ("scale", "gate"), ()]


@pytest.mark.parametrize("T,d", SIZES)
def test_forward_sizes(T, d):
    require_gpu()
    say(f"block_norm T={T} d={d}")
    check_forward(make(T, d))


@pytest.mark.parametrize("parts", PARTS)
@pytest.mark.parametrize("h,y,x,w", [("bf16", "f32", "bf16", "bf16"), ("f32", "bf16", "bf16", "f32"), ("f32", "f32", "f32", "f32"),
                                     ("bf16", "bf16", "f32", "bf16")])
def test_forward_types_and_parts(h, y, x, w, parts):
    require_gpu()
    say(f"block_norm {h} {y} {x} {w} {parts}")
    check_forward(make(11, 1304, h, y, x, w, parts=parts), x=x)


@pytest.mark.parametrize("h,x", [("bf16", "bf16"), ("f32", "f32")])
def test_forward_without_a_block(h, x):
    require_gpu()
    say(f"block_norm alone {h} {x}")
    p = make(21, 776, h, x=x, parts=("pre",))
    p["y"] = None
    check_forward(p, x=x, alpha=1.0)


@pytest.mark.parametrize("T,d,k", [(1, 2048, 8), (5, 264, 3), (33, 4096, 2), (2, 16384, 32), (1, 64, 1)])
@pytest.mark.parametrize("y", ["f32", "bf16"])
def test_forward_combines_slots(T, d, k, y):
    """Repeated rows, dropped slots (-1), rows out of range, a token without any
    slot; a dropped slot's weight and the rows nobody names are not looked at."""
    require_gpu()
    say(f"block_norm slots T={T} d={d} k={k} {y}")
    p = make(T, d, y=y, rows=T * k + 2)
    g = torch.Generator(device="cuda")
    g.manual_seed(5)
    row = torch.randint(0, T * k, (T, k), device="cuda", generator=g, dtype=torch.int32)
    w = torch.softmax(torch.randn(T, k, device="cuda", generator=g), 1)
    if k > 1:
        row[0, 0], w[0, 0] = -1, float("nan")
    if T > 1:
        row[1] = T * k + 2  # out of range
    p["y"][T * k:] = float("nan")
    check_forward(p, slot_row=row, slot_weights=w)


def test_empty_token_without_norm_factor():
    """A token without slots has y = 0: the post norm divides by sqrt(eps), and
    the stream passes through."""
    require_gpu()
    p = make(2, 512, y="f32")
    row = torch.full((2, 4), -1, device="cuda", dtype=torch.int32)
    h_out, _ = lb.block_norm(p["h"], p["y"], **weights(p), slot_row=row, slot_weights=torch.ones(2, 4, device="cuda"))
    assert torch.equal(h_out, p["h"])


def test_no_rows_to_combine():
    require_gpu()
    p = make(2, 512, y="f32", rows=4)
    row = torch.zeros(2, 4, device="cuda", dtype=torch.int32)
    h_out, _ = lb.block_norm(p["h"], p["y"][:0], **weights(p), slot_row=row, slot_weights=torch.ones(2, 4, device="cuda"))
    assert h_out is not p["h"] and torch.equal(h_out, p["h"])


def test_in_place_and_given_outputs():
    require_gpu()
    p = make(9, 1024)
    ref = lb.block_norm(p["h"], p["y"], **weights(p))
    h, x = p["h"].clone(), torch.empty_like(p["h"])
    got = lb.block_norm(h, p["y"], **weights(p), h_out=h, x=x)
    assert got[0] is h and got[1] is x and torch.equal(h, ref[0]) and torch.equal(x, ref[1])


def test_extreme_values():
    """Zero rows, infinities and NaN stay in their own row."""
    require_gpu()
    p = make(5, 256, "f32", "f32", "f32", "f32")
    p["h"][1] = 0
    p["y"][1] = 0
    p["y"][2, 7] = float("inf")
    p["h"][3, 9] = float("nan")
    h_out, x = lb.block_norm(p["h"], p["y"], **weights(p), x_dtype=torch.float32)
    assert torch.equal(h_out[1], torch.zeros_like(h_out[1])) and torch.equal(x[1], torch.zeros_like(x[1]))
    for r in (0, 4):
        assert torch.isfinite(h_out[r]).all() and torch.isfinite(x[r]).all()
    assert torch.isnan(h_out[2, 7]) and torch.isnan(x[3]).all()


def check_backward(p, alpha=0.9, eps=1e-5, dh_out=True):
    g = lb.block_norm_backward(p["h"], p["y"], p["dx"] if p["w_pre"] is not None else None, p["dh_out"] if dh_out else None,
                               **weights(p), residual_scale=alpha, eps=eps)
    torch.cuda.synchronize()
    ref = O.block_norm_grads(host(p["h"]), host(p["y"]), host(p["dx"]), host(p["dh_out"]) if dh_out else None,
                             **{n: host(v) for n, v in weights(p).items()}, residual_scale=float(np.float32(alpha)),
                             eps=float(np.float32(eps)))
    got = {n: v for n, v in g._asdict().items() if v is not None}
    assert set(got) == set(ref)
    for n, (r, mag) in ref.items():
        within(n, got[n], r, mag)
    return g


@pytest.mark.parametrize("T,d", SIZES + [(600, 64), (1025, 520), (2500, 2048)])
def test_backward_sizes(T, d):
    require_gpu()
    say(f"block_norm_backward T={T} d={d}")
    check_backward(make(T, d))


@pytest.mark.parametrize("parts", PARTS)
@pytest.mark.parametrize("h,y,x,w", [("bf16", "f32", "bf16", "bf16"), ("f32", "bf16", "bf16", "f32"), ("f32", "f32", "f32", "f32")])
def test_backward_types_and_parts(h, y, x, w, parts):
    require_gpu()
    say(f"block_norm_backward {h} {y} {x} {w} {parts}")
    check_backward(make(13, 1304, h, y, x, w, parts=parts))
    check_backward(make(13, 4232, h, y, x, w, parts=parts), dh_out="pre" not in parts)


def test_backward_without_a_block():
    require_gpu()
    for T, d in ((21, 776), (5, 2304), (3, 8192)):
        p = make(T, d, parts=("pre",))
        p["y"] = None
        check_backward(p)


def test_backward_of_no_tokens_clears_weight_gradients():
    require_gpu()
    p = make(4, 64)
    e = lambda n: p[n][:0].contiguous()  # noqa: E731
    g = lb.block_norm_backward(e("h"), e("y"), e("dx"), None, w_pre=p["w_pre"], w_post=p["w_post"], scale=p["scale"])
    torch.cuda.synchronize()
    for v in (g.dw_pre, g.dw_post, g.dscale):
        assert torch.equal(v, torch.zeros_like(v))
    assert lb.block_norm(e("h"), e("y"), w_pre=p["w_pre"])[1].shape == (0, 64)


@pytest.mark.parametrize("T,d,h", [(3, 64, "f32"), (5, 512, "bf16"), (3, 1000, "bf16"), (257, 2048, "f32")])
def test_backward_with_eps_0(T, d, h):
    """The rows that a workgroup has to spare add nothing to the weights' gradients,
    also where their norm factor would be infinite."""
    require_gpu()
    check_backward(make(T, d, h, "bf16", "bf16"), eps=0.0)


def test_backward_agrees_with_differences():
    """The gradients against differences of the library's own forward, fp32,
    loss = sum(a h_out) + sum(b x): central differences with step s of a smooth
    loss of size L are off by about 2^-24 L / s + s^2; with s = 2^-6, L ~ 50 and
    gradients of order 1 that is below 1e-2."""
    require_gpu()
    T, d = 3, 64
    p = make(T, d, "f32", "f32", "f32", "f32", seed=3)
    a, b = p["dh_out"], p["dx"]
    kw = dict(residual_scale=0.8, eps=1e-4)

    def loss(**ch):
        q = dict(p, **ch)
        ho, x = lb.block_norm(q["h"], q["y"], **weights(q), x_dtype=torch.float32, **kw)
        return ((a.double() * ho.double()).sum() + (b.double() * x.double()).sum()).item()

    ho, _ = lb.block_norm(p["h"], p["y"], **weights(p), x_dtype=torch.float32, **kw)
    g = lb.block_norm_backward(ho, p["y"], b, a, **weights(p), **kw)
    s = 2.0 ** -6
    for name, grad in (("h", g.dh), ("y", g.dy), ("gate", g.dgate), ("w_pre", g.dw_pre), ("w_post", g.dw_post), ("scale", g.dscale)):
        for at in (0, 5, p[name].numel() - 1) if p[name].numel() > 5 else range(p[name].numel()):
            up, dn = p[name].clone(), p[name].clone()
            up.view(-1)[at] += s
            dn.view(-1)[at] -= s
            num = (loss(**{name: up}) - loss(**{name: dn})) / (2 * s)
            assert abs(num - grad.view(-1)[at].item()) <= 1e-2 * max(1.0, abs(num)), (name, at)


def test_same_bits_on_every_run_and_in_a_graph():
    """Repeated calls and graph replays (with other work between them) give the
    same bits; dh may be dh_out."""
    require_gpu()
    p = make(700, 1024)
    ref_f = lb.block_norm(p["h"], p["y"], **weights(p))
    ref_b = lb.block_norm_backward(p["h"], p["y"], p["dx"], p["dh_out"], **weights(p))
    dh = p["dh_out"].clone()
    assert lb.block_norm_backward(p["h"], p["y"], p["dx"], dh, **weights(p), dh=dh).dh is dh
    assert torch.equal(dh, ref_b.dh)
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(st):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=st):
            f = lb.block_norm(p["h"], p["y"], **weights(p))
            b = lb.block_norm_backward(p["h"], p["y"], p["dx"], p["dh_out"], **weights(p))
    for _ in range(3):
        for v in (*f, *b):
            v.fill_(7)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for v, r in zip((*f, *b), (*ref_f, *ref_b)):
            assert torch.equal(v, r)


def test_other_stream():
    require_gpu()
    p = make(300, 2048)
    ref = lb.block_norm_backward(p["h"], p["y"], p["dx"], p["dh_out"], **weights(p))
    torch.cuda.synchronize()
    st = torch.cuda.Stream()
    got = lb.block_norm_backward(p["h"], p["y"], p["dx"], p["dh_out"], **weights(p), stream=st)
    st.synchronize()
    for v, r in zip(got, ref):
        assert torch.equal(v, r)


def test_offsets_past_32_bits():
    """Rows whose byte and element offsets pass 2^32 and 2^31."""
    require_gpu()
    d = 8192
    T = (1 << 31) // d + 3
    h = torch.zeros(T, d, dtype=torch.bfloat16, device="cuda")
    p = make(3, d)
    h[-3:] = p["h"]
    w = p["w_pre"]
    _, x = lb.block_norm(h, w_pre=w)
    assert torch.equal(x[-3:], lb.block_norm(p["h"], w_pre=w)[1]) and not x[:3].any()
    g = lb.block_norm_backward(h, None, x, w_pre=w)
    ref = lb.block_norm_backward(p["h"], None, x[-3:].contiguous(), w_pre=w)
    assert torch.equal(g.dh[-3:], ref.dh)


@pytest.mark.parametrize("bad", [dict(y=torch.float16), dict(gate=torch.bfloat16), dict(h_out=torch.float32)])
def test_wrapper_refuses_types(bad):
    require_gpu()
    p = make(4, 64)
    kw = weights(p)
    h_out = torch.empty_like(p["h"])
    if "y" in bad:
        p["y"] = p["y"].to(bad["y"])
    if "gate" in bad:
        kw["gate"] = kw["gate"].to(bad["gate"])
    if "h_out" in bad:
        h_out = h_out.to(bad["h_out"])
    with pytest.raises(ValueError):
        lb.block_norm(p["h"], p["y"], **kw, h_out=h_out)


def test_wrapper_refuses_shapes():
    require_gpu()
    p = make(4, 64)
    with pytest.raises(ValueError):
        lb.block_norm(p["h"].t(), w_pre=p["w_pre"])
    with pytest.raises(ValueError):
        lb.block_norm(p["h"], p["y"][:3], w_pre=p["w_pre"])
    with pytest.raises(ValueError):
        lb.block_norm(p["h"], w_pre=p["w_pre"].float(), y=p["y"], w_post=p["w_post"])
    with pytest.raises(ValueError):
        lb.block_norm(p["h"], p["y"], w_pre=p["w_pre"], gate=p["gate"].cpu())
    with pytest.raises(lx.LorexError) as e:
        lb.block_norm(p["h"][:, :60].contiguous(), w_pre=p["w_pre"][:60].contiguous())
    assert e.value.status == lx.LX_ERR_UNSUPPORTED

"""The MoE block with its activations in 8 bits or not rounded, and a training step with
dropout, as a run of the operators together.

Bounds, fixed before the first run. In 8 bits: the norm's and SwiGLU's values differ from
the oracle's codes only next to a midpoint between two codes, within fp32's error of it
(less than 1 in 1000 values), then by one step, an eighth of the value at most: 4e-3 of
a row's norm; the sums after it are in fp32 and h_out is rounded to bf16: 1e-2 in the
2-norm, 0.1 of the RMS for any value. Not rounded: bf16's 2^-8 of a value, and 1e-4 of the
RMS for the fp32 sums (2048 terms at most, 2^-24 each, of ten times the result's size)."""
import os
import subprocess
import sys

import numpy as np
import pytest
import torch

from oracle import block as O
from paper_2608_07814_amd import block as lb
from gpu_util import require_gpu, say

pytestmark = pytest.mark.gpu


def host(t):
    return t.detach().cpu().double().numpy()


def deq(q):
    return O.dequantize(q.codes.cpu().numpy(), q.scales.cpu().numpy(), q.K)


def make(T, E, d, f, seed=0):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed + T)
    r = lambda *s: torch.randn(*s, device="cuda", generator=g)  # noqa: E731
    ex = lb.mx4_experts((r(E, f, d) * d ** -0.5).bfloat16(), (r(E, f, d) * d ** -0.5).bfloat16(), (r(E, d, f) * d ** -0.5).bfloat16())
    w_pre, w_post, w_next, scale = (1 + 0.1 * r(4, d)).bfloat16()
    return dict(h=r(T, d).bfloat16(), w_pre=w_pre, w_r=r(E, d).bfloat16(), experts=ex), dict(
        w_post=w_post, scale=scale, gate=torch.sigmoid(r(T)), residual_scale=0.5, w_next=w_next)


@pytest.mark.parametrize("T,E,d,f,k", [(1, 8, 128, 64, 2), (7, 16, 256, 96, 4), (64, 8, 192, 128, 8), (300, 32, 256, 200, 3), (5, 64, 1024, 72, 8)])
@pytest.mark.parametrize("activations", ["mx8", "full"])
def test_block_matches_oracle(T, E, d, f, k, activations):
    require_gpu()
    if activations == "full":
        T = min(T, lb.MOE_FEW_MAX_T)
    say(f"mx4_moe_block {activations} T={T} E={E} d={d} f={f} k={k}")
    a, more = make(T, E, d, f)
    out = lb.mx4_moe_block(*a.values(), k, **more, balance_coef=1.0, activations=activations)
    torch.cuda.synchronize()
    ids, wt = out.topk_ids.cpu().numpy(), host(out.topk_weights)
    x = O.block_norm(host(a["h"]), None, host(a["w_pre"]))[1]
    assert np.max(np.abs(host(out.x) - x)) <= 2.0 ** -7 * np.max(np.abs(x))
    gu, dn = deq(a["experts"].gate_up), deq(a["experts"].down)
    round8 = lambda v: O.dequantize8(*O.quantize8(v)[:2], v.shape[1])  # noqa: E731
    x = round8(x) if activations == "mx8" else host(out.x)
    y = np.zeros((T, d))
    for t in range(T):
        for j in range(k):
            v = O.silu_mul((gu[ids[t, j]] @ x[t])[None])
            y[t] += wt[t, j] * (dn[ids[t, j]] @ (round8(v) if activations == "mx8" else v)[0])
    w = {n: host(v) for n, v in more.items() if n in ("w_post", "scale", "gate")}
    ref_h, ref_x, _, _ = O.block_norm(host(a["h"]), y, host(more["w_next"]), **w, residual_scale=0.5, eps=float(np.float32(1e-6)))
    for name, got, ref in (("h_out", out.h_out, ref_h), ("x_next", out.x_next, ref_x)):
        diff, rms = np.abs(host(got) - ref), np.sqrt(np.mean(ref * ref))
        say(f"  {name}: rel {np.linalg.norm(diff) / np.linalg.norm(ref):.2e}, worst {np.max(diff) / rms:.2e}")
        if activations == "full":
            assert np.all(diff <= 2.0 ** -8 * np.abs(ref) + 1e-4 * rms)
        else:
            assert np.linalg.norm(diff) <= 1e-2 * np.linalg.norm(ref) and np.max(diff) <= 0.1 * rms
    loss, counts, _, n, _, _ = O.balance(host(out.logits), ids)
    assert np.array_equal(out.balance.counts.cpu().numpy(), counts) and n == T


@pytest.mark.parametrize("activations,T", [("mx8", 40), ("mx8", 3), ("full", 1), ("full", 33)])
def test_block_in_a_graph(activations, T):
    """Captured once, replayed on other tokens in the same memory."""
    require_gpu()
    a, more = make(T, 16, 256, 128)
    run = lambda: lb.mx4_moe_block(*a.values(), 4, **more, activations=activations)  # noqa: E731
    run()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        with torch.cuda.graph(graph, stream=side):
            got = run()
    torch.cuda.current_stream().wait_stream(side)
    for i in range(3):
        a["h"].copy_(torch.randn(T, 256, device="cuda"))
        graph.replay()
        ref = run()
        torch.cuda.synchronize()
        for name in ("h_out", "x_next", "x", "topk_ids"):
            assert torch.equal(getattr(got, name), getattr(ref, name)), (i, name)


def test_a_training_steps_norms():
    """Forward with dropout into the next block's input, backward through both norms, and
    the same with the block's input in 8 bits: its gradient passes through the rounding."""
    require_gpu()
    g = torch.Generator(device="cuda")
    g.manual_seed(4)
    r = lambda *s: torch.randn(*s, device="cuda", generator=g)  # noqa: E731
    T, d, p = 21, 264, 0.25
    h, y, w_pre, w_post, w_next = r(T, d), r(T, d), 1 + 0.1 * r(d), 1 + 0.1 * r(d), 1 + 0.1 * r(d)
    dx_in, dx_next, dh_next = r(T, d), r(T, d), r(T, d)  # of the block's input, the next one's, the stream
    rng = torch.tensor([77, 3], device="cuda")
    keep = O.dropout_keep(T, d, p, 77, 3)
    _, x8 = lb.block_norm_mx8(h, w_pre=w_pre)
    h1, _ = lb.block_norm_dropout(h, y, p, rng, w_pre=w_next, w_post=w_post)
    after = lb.block_norm_dropout_backward(h1, y, dx_next, dh_next, p, rng, w_pre=w_next, w_post=w_post)
    before = lb.block_norm_backward(h, None, dx_in, after.dh, w_pre=w_pre)
    eps = float(np.float32(1e-6))
    assert np.linalg.norm(host(lb.mx8_dequantize(x8, torch.float32)) - O.block_norm(host(h), None, host(w_pre), eps=eps)[1]) <= 2.0 ** -4 * np.linalg.norm(
        O.block_norm(host(h), None, host(w_pre), eps=eps)[1])
    H, Y, WP, WO, WN = (host(v) for v in (h, y, w_pre, w_post, w_next))

    def loss(H, Y, WP, WO, WN):
        x = O.block_norm(H, None, WP, eps=eps)[1]
        o, n = O.block_norm(H, Y, WN, WO, eps=eps, keep=keep)[:2]
        return (x * host(dx_in)).sum() + (o * host(dh_next)).sum() + (n * host(dx_next)).sum()

    rng64, args = np.random.default_rng(0), [H, Y, WP, WO, WN]
    for i, got in enumerate((before.dh, after.dy, before.dw_pre, after.dw_post, after.dw_pre)):
        v, step = rng64.normal(size=args[i].shape), 1e-5
        plus, minus = list(args), list(args)
        plus[i], minus[i] = args[i] + step * v, args[i] - step * v
        diff = (loss(*plus) - loss(*minus)) / (2 * step)
        # fp32: 256 * 2^-24 of the terms' magnitudes each in two norms
        assert abs(diff - (host(got) * v).sum()) <= 4 * 256 * 2.0 ** -24 * np.abs(host(got) * v).sum() + 1e-5, i


def test_refusals():
    require_gpu()
    a, more = make(65, 8, 128, 64)
    with pytest.raises(ValueError):
        lb.mx4_moe_block(*a.values(), 2, **more, activations="full")
    with pytest.raises(ValueError):
        lb.mx4_moe_block(*a.values(), 2, **more, activations="bf16")


def test_block_of_no_tokens():
    require_gpu()
    a, more = make(2, 8, 128, 64)
    a["h"], more["gate"] = a["h"][:0], more["gate"][:0]
    for activations in ("mx8", "full"):
        out = lb.mx4_moe_block(*a.values(), 2, **more, balance_coef=1.0, activations=activations)
        assert out.h_out.shape == out.x.shape == out.x_next.shape == (0, 128) and out.topk_ids.shape == (0, 2)


@pytest.mark.parametrize("more", [["--activations", "mx8", "--decode-activations", "full", "--dropout", "0.1"],
                                  ["--activations", "mx8", "--decode-activations", "mx8"]])
def test_example_runs(more):
    require_gpu()
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    r = subprocess.run([sys.executable, os.path.join(root, "examples", "moe_block.py"), "--experts", "16", "--d", "256", "--f", "128",
                        "--k", "2", "--tokens", "333", "--decode", "3", *more], capture_output=True, text=True, timeout=100)
    assert r.returncode == 0, r.stderr[-2000:]
    assert [line.split(":")[0] for line in r.stdout.splitlines()] == ["prompt", "decode", "training"]

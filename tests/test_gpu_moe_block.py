"""The MoE block with its experts in 4 bits against the fp64 oracle of its parts.

Bound, fixed before the first run: with the block's own input x, ids and weights
given, the gate and up projections are sums of exact products whose fp32 and bf16
rounding is the oracle's but for ties, so the rounded activations differ from the
oracle's only where a value lies within about 2^-8 of a midpoint between two bf16
neighbours, and then by one 4-bit step: less than 1 in 1000 values, 0.2 of the
value, 6e-3 of a row's norm. The sums after it are in fp32 and h_out is rounded
to bf16 (2^-9 on average): 1e-2 in the 2-norm, and 0.1 of the RMS for any value."""
import subprocess
import sys
import os

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


def bf16(a):
    return torch.from_numpy(a.astype(np.float32)).bfloat16().double().numpy()


@pytest.mark.parametrize("T,E,d,f,k", [(1, 8, 128, 64, 2), (7, 16, 256, 96, 4), (70, 8, 192, 128, 8), (300, 32, 256, 200, 3)])
def test_block_matches_oracle(T, E, d, f, k):
    require_gpu()
    say(f"mx4_moe_block T={T} E={E} d={d} f={f} k={k}")
    g = torch.Generator(device="cuda")
    g.manual_seed(T)
    r = lambda *s: torch.randn(*s, device="cuda", generator=g)  # noqa: E731
    ex = lb.mx4_experts((r(E, f, d) * d ** -0.5).bfloat16(), (r(E, f, d) * d ** -0.5).bfloat16(), (r(E, d, f) * d ** -0.5).bfloat16())
    h, w_r = r(T, d).bfloat16(), r(E, d).bfloat16()
    w_pre, w_post, w_next, scale = (1 + 0.1 * r(4, d)).bfloat16()
    gate = torch.sigmoid(r(T))
    out = lb.mx4_moe_block(h, w_pre, w_r, ex, k, w_post=w_post, scale=scale, gate=gate, residual_scale=0.5, w_next=w_next, balance_coef=1.0)
    torch.cuda.synchronize()
    x = host(out.x)
    assert np.max(np.abs(x - O.block_norm(host(h), None, host(w_pre))[1])) <= 2.0 ** -7 * np.max(np.abs(x))
    ids, wt = out.topk_ids.cpu().numpy(), host(out.topk_weights)
    # the experts in fp64 from the 4-bit values
    xq = O.dequantize(*O.quantize(x)[:2], d)
    gu, dn = deq(ex.gate_up), deq(ex.down)
    y = np.zeros((T, d))
    for t in range(T):
        for j in range(k):
            e = ids[t, j]
            v = bf16(gu[e] @ xq[t])[None]
            a = O.silu_mul(v)
            y[t] += wt[t, j] * (dn[e] @ O.dequantize(*O.quantize(a)[:2], f)[0])
    ref_h, ref_x, _, _ = O.block_norm(host(h), y, host(w_next), host(w_post), host(scale), host(gate), 0.5, float(np.float32(1e-6)))
    for name, got, ref in (("h_out", out.h_out, ref_h), ("x_next", out.x_next, ref_x)):
        diff = host(got) - ref
        rel, worst = np.linalg.norm(diff) / np.linalg.norm(ref), np.max(np.abs(diff)) / np.sqrt(np.mean(ref * ref))
        say(f"  {name}: rel {rel:.2e}, worst {worst:.2e}")
        assert rel <= 1e-2 and worst <= 0.1
    loss, counts, _, n, _, _ = O.balance(host(out.logits), ids)
    assert np.array_equal(out.balance.counts.cpu().numpy(), counts) and n == T
    assert abs(out.balance.loss.item() - loss) <= 1e-4 * loss


def test_block_of_no_tokens():
    require_gpu()
    g = torch.Generator(device="cuda")
    g.manual_seed(2)
    r = lambda *s: torch.randn(*s, device="cuda", generator=g).bfloat16()  # noqa: E731
    E, d, f, k = 8, 128, 64, 2
    ex = lb.mx4_experts(r(E, f, d), r(E, f, d), r(E, d, f))
    out = lb.mx4_moe_block(r(0, d), r(d), r(E, d), ex, k, w_next=r(d), balance_coef=1.0)
    torch.cuda.synchronize()
    assert out.h_out.shape == out.x_next.shape == out.x.shape == (0, d) and out.h_out.dtype == torch.bfloat16
    assert out.topk_ids.shape == out.topk_weights.shape == (0, k) and out.logits.shape == (0, E)
    assert out.balance.loss.item() == 0 and not out.balance.counts.any()


def test_block_refuses_what_does_not_fit():
    require_gpu()
    r = lambda *s: torch.randn(*s, device="cuda").bfloat16()  # noqa: E731
    E, d, f = 8, 128, 64
    ex = lb.mx4_experts(r(E, f, d), r(E, f, d), r(E, d, f))
    other = lb.mx4_experts(r(E, f, d), r(E, f, d), r(4, d, f))
    for h, w_r, e in ((r(3, d), r(E + 4, d), ex), (r(3, d), r(E, 2 * d), ex), (r(3, 2 * d), r(E, 2 * d), ex),
                      (r(3, d), r(E, d).cpu(), ex), (r(3, d), r(E, d), lb.Mx4Experts(ex.gate_up, other.down)),
                      (r(3, d), r(E, d), lb.Mx4Experts(ex.down, ex.down))):
        with pytest.raises(ValueError):
            lb.mx4_moe_block(h, r(d), w_r, e, 2)


def test_given_workspaces():
    """A workspace that is not plain bytes on the call's GPU is refused; one that is
    large enough is used."""
    require_gpu()
    T, E, k, d = 3000, 64, 2, 256
    lg = torch.randn(T, E, device="cuda")
    ids = torch.topk(lg, k, dim=1).indices.int()
    need = lb.lib().lx_balance_loss_workspace_bytes(T, E)
    assert need > 0
    ref = lb.balance_loss(lg, ids)
    got = lb.balance_loss(lg, ids, workspace=torch.empty(need, dtype=torch.uint8, device="cuda"))
    assert torch.equal(got.loss, ref.loss) and torch.equal(got.counts, ref.counts)
    h = torch.randn(T, d, device="cuda")
    big = lb.lib().lx_block_norm_backward_workspace_bytes(T, d)
    for n, call in ((need, lambda w: lb.balance_loss(lg, ids, workspace=w)),
                    (big, lambda w: lb.block_norm_backward(h, None, h, w_pre=h[0], workspace=w))):
        for w in (torch.empty(n, dtype=torch.uint8), torch.empty(n, dtype=torch.float32, device="cuda"),
                  torch.empty(1, dtype=torch.uint8, device="cuda").expand(n),
                  torch.empty(2 * n, dtype=torch.uint8, device="cuda")[::2]):
            with pytest.raises(ValueError):
                call(w)


def test_example_runs():
    require_gpu()
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    r = subprocess.run([sys.executable, os.path.join(root, "examples", "moe_block.py"), "--experts", "16", "--d", "256", "--f", "128",
                        "--k", "2", "--tokens", "333", "--decode", "3"], capture_output=True, text=True, timeout=100)
    assert r.returncode == 0, r.stderr[-2000:]
    assert [line.split(":")[0] for line in r.stdout.splitlines()] == ["prompt", "decode", "training"]

"""The experts' layer for a few tokens on the GPU against a fp64 form.

Bounds, fixed before the first run: a sum of n fp32 products is off by at most 2^-24 n
of its terms' magnitudes; SwiGLU and the router's weight add 2^-24 * 16 (1 + |gate|) of
the hidden value; with a bf16 output the hidden values are off by 2^-16 and the result
by 2^-8 (with fp32 by 2^-24)."""
import numpy as np
import pytest
import torch

from oracle import block as O
from paper_2608_07814_amd import block as lb
from paper_2608_07814_amd import lorex as lx
from gpu_util import require_gpu, say

pytestmark = pytest.mark.gpu

DT = {"f32": torch.float32, "bf16": torch.bfloat16}
U = 2.0 ** -24


def host(t):
    return t.detach().cpu().double().numpy()


def weights4(G, N, K, rng, spread=2):
    Kp = O.padded(K)
    codes = rng.integers(0, 256, size=(G, N, Kp // 2)).astype(np.uint8)
    scales = rng.integers(122 - spread, 123 + spread, size=(G, N, Kp // 32)).astype(np.uint8)
    codes[:, :, K // 2:] = 0
    scales[:, :, -(-K // 32):] = 0
    return lb.Mx4(torch.from_numpy(codes).cuda(), torch.from_numpy(scales).cuda(), K)


def layer(E, d, f, seed=0, spread=2):
    rng = np.random.default_rng(seed + E + d + f)
    return lb.Mx4Experts(weights4(E, 2 * f, d, rng, spread), weights4(E, d, f, rng, spread))


def values(q):
    return O.dequantize(q.codes.cpu().numpy(), q.scales.cpu().numpy(), q.K)


def routing(T, k, E, seed=0):
    rng = np.random.default_rng(seed + 31 * T + k)
    ids = np.stack([rng.permutation(E)[:k] for _ in range(T)]).astype(np.int32) if k <= E else rng.integers(0, E, (T, k)).astype(np.int32)
    return torch.from_numpy(ids).cuda(), torch.from_numpy(rng.random((T, k)).astype(np.float32)).cuda()


def reference(x, ids, w, ex, out):
    """(result, bound) in fp64."""
    d, f = ex.gate_up.K, ex.down.K
    gu, dn = values(ex.gate_up), values(ex.down)
    X, I, W = host(x), ids.cpu().numpy(), host(w)
    ref, tol = np.zeros((len(X), d)), np.zeros((len(X), d))
    n = 0
    for t in range(len(X)):
        for j in range(I.shape[1]):
            e = I[t, j]
            if not 0 <= e < len(dn):
                continue
            n += 1
            z, mag = gu[e] @ X[t], np.abs(gu[e]) @ np.abs(X[t])
            g, u, dg, du = z[:f], z[f:], U * d * mag[:f], U * d * mag[f:]
            with np.errstate(over="ignore"):
                s = g / (1 + np.exp(-g))
            h = s * u * W[t, j]
            dh = np.abs(W[t, j]) * (1.1 * dg * np.abs(u) + np.abs(s) * du) + 16 * U * (1 + np.abs(g)) * np.abs(h)
            if out == torch.bfloat16:
                dh = dh + 2.0 ** -16 * np.abs(h)
            ref[t] += dn[e] @ h
            tol[t] += np.abs(dn[e]) @ (dh + U * f * I.shape[1] * np.abs(h))
    unit = 2.0 ** -8 if out == torch.bfloat16 else U
    return ref, tol + unit * np.abs(ref) + 1e-36


def check(x, ids, w, ex, out=torch.float32, **kw):
    got = lb.mx4_moe_few(x, ids, w, ex, out_dtype=out, **kw)
    torch.cuda.synchronize()
    ref, tol = reference(x, ids, w, ex, out)
    err = np.abs(host(got) - ref)
    # (where |ref| + tol passes fp32's largest value, 2^128 (1 - 2^-24), an fp32 sum within
    # tol of ref may be one that fp32 does not hold: it is then infinite)
    past = ~np.isfinite(host(got)) & (np.abs(ref) + tol >= 2.0 ** 128 * (1 - 2.0 ** -24))
    bad = ~(err <= tol) & ~past
    assert got.dtype == out and not bad.any(), f"{bad.sum()} of {err.size} off, {np.max((err / tol)[~past]):.3g} of the bound"
    return got


def tokens(T, d, dtype, seed=0):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed + T + d)
    return torch.randn(T, d, device="cuda", generator=g).to(DT[dtype])


SIZES = [(1, 1, 1, 8, 8), (1, 8, 128, 256, 64), (1, 2, 8, 2048, 768), (2, 3, 5, 136, 40), (5, 2, 8, 264, 1000), (16, 4, 16, 512, 96),
         (17, 1, 2, 128, 128), (33, 8, 64, 640, 72), (61, 8, 128, 256, 200), (64, 6, 6, 120, 24), (64, 32, 40, 64, 32), (3, 2, 300, 64, 48),
         (64, 1, 1, 72, 520), (40, 2, 3, 1032, 8), (64, 32, 2100, 64, 8), (9, 3, 7, 24, 4096),
         (37, 5, 20, 2056, 776), (30, 8, 9, 768, 1544)]


@pytest.mark.parametrize("T,k,E,d,f", SIZES)
@pytest.mark.parametrize("x,out", [("bf16", "bf16"), ("bf16", "f32"), ("f32", "f32"), ("f32", "bf16")])
def test_sizes_and_types(T, k, E, d, f, x, out):
    require_gpu()
    say(f"moe_few T={T} k={k} E={E} d={d} f={f} {x} {out}")
    ids, w = routing(T, k, E)
    check(tokens(T, d, x), ids, w, layer(E, d, f), DT[out])


def test_slots_without_experts_and_experts_named_twice():
    require_gpu()
    E, d, f = 12, 264, 104
    ids, w = routing(9, 4, E)
    ids[0] = -1                                 # nothing at all
    ids[1] = torch.tensor([3, 3, 3, 3])         # one expert four times
    ids[2] = torch.tensor([E, 2, -5, 2])        # out of range, and twice
    ids[3] = torch.tensor([1 << 30, -1 << 30, E - 1, 0])
    ids[7] = ids[8]                             # the same experts as another token
    w[2, 0] = float("nan")                      # (of a slot that is not there)
    for T in (9, 4, 3):                         # by experts and by slots
        for out in DT.values():
            wc = torch.where((ids[:T] < 0) | (ids[:T] >= E), torch.zeros_like(w[:T]), w[:T])
            x = tokens(T, d, "f32")
            got = lb.mx4_moe_few(x, ids[:T].contiguous(), w[:T].contiguous(), layer(E, d, f), out_dtype=out)
            ref, tol = reference(x, ids[:T], wc, layer(E, d, f), out)
            assert np.all(np.abs(host(got) - ref) <= tol) and not got[0].any()


def test_all_tokens_on_one_expert():
    require_gpu()
    for T in (16, 17, 63, 64):
        ids, w = routing(T, 2, 64)
        ids[:, 0], ids[:, 1] = 5, -1
        check(tokens(T, 200, "bf16"), ids, w, layer(64, 200, 136), torch.bfloat16)


@pytest.mark.parametrize("spread", [20, 60])
def test_scales_of_very_different_sizes(spread):
    """Blocks whose scales differ by up to 2^(4 spread / 2): bf16 holds every weight."""
    require_gpu()
    ex = layer(4, 264, 136, spread=spread)
    ids, w = routing(5, 2, 4)
    x = tokens(5, 264, "f32") * 2.0 ** -20
    check(x, ids, w, ex)


def test_infinite_and_nan_values_stay_with_their_tokens():
    require_gpu()
    E, d, f = 6, 256, 64
    ex = layer(E, d, f)
    ids, w = routing(8, 2, E)
    ids[:, 0], ids[:, 1] = torch.arange(8, device="cuda") % 3, 3
    x = tokens(8, d, "f32")
    ref = lb.mx4_moe_few(x, ids, w, ex)
    y = x.clone()
    y[2, 7], y[5, 100] = float("inf"), float("nan")
    got = lb.mx4_moe_few(y, ids, w, ex)
    clean = [0, 1, 3, 4, 6, 7]
    assert torch.equal(got[clean], ref[clean]) and not torch.isfinite(got[[2, 5]]).any()
    ex.gate_up.scales[1, 5, 3] = 255            # a NaN block of expert 1: tokens 1, 4, 7
    got = lb.mx4_moe_few(x, ids, w, ex)
    clean = [0, 2, 3, 5, 6]
    assert torch.equal(got[clean], ref[clean]) and torch.isnan(got[[1, 4, 7]]).all()


def test_given_output_workspace_stream_and_repeats():
    """A workspace full of ones, used again by other calls; the same bits each time; a
    stream of its own."""
    require_gpu()
    ex = layer(16, 512, 256)
    n = lb.lib().lx_mx4_moe_few_workspace_bytes(64, 4, 16, 512, 256)
    ws = torch.full((n,), 255, dtype=torch.uint8, device="cuda")
    side = torch.cuda.Stream()
    for T in (64, 3, 17):
        ids, w = routing(T, 4, 16)
        x = tokens(T, 512, "bf16")
        out = torch.full((T, 512), float("nan"), device="cuda")
        assert check(x, ids, w, ex, out=torch.float32, workspace=ws) is not None
        ref = lb.mx4_moe_few(x, ids, w, ex, out=out)
        assert ref is out
        side.wait_stream(torch.cuda.current_stream())
        again = lb.mx4_moe_few(x, ids, w, ex, stream=side, workspace=ws)
        torch.cuda.current_stream().wait_stream(side)
        assert torch.equal(again, out)
    need = lb.lib().lx_mx4_moe_few_workspace_bytes(17, 4, 16, 512, 256)
    with pytest.raises(lx.LorexError):
        lb.mx4_moe_few(x, ids, w, ex, workspace=ws[:need - 1])


def test_two_captured_graphs_share_a_workspace():
    require_gpu()
    ex = layer(16, 512, 256)
    ws = torch.zeros(lb.lib().lx_mx4_moe_few_workspace_bytes(64, 4, 16, 512, 256), dtype=torch.uint8, device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    made = []
    for T in (5, 40):
        ids, w = routing(T, 4, 16)
        x = tokens(T, 512, "bf16")
        graph, out = torch.cuda.CUDAGraph(), torch.empty(T, 512, device="cuda")
        with torch.cuda.stream(side):
            with torch.cuda.graph(graph, stream=side):
                lb.mx4_moe_few(x, ids, w, ex, out=out, workspace=ws)
        made.append((graph, out, x, ids, w))
    torch.cuda.current_stream().wait_stream(side)
    for i in range(3):
        for graph, out, x, ids, w in made:
            ids.copy_(ids.roll(1, 0))           # other routing in the same memory
            graph.replay()
            assert torch.equal(out, lb.mx4_moe_few(x, ids, w, ex))


def test_empty_and_refusals():
    require_gpu()
    ex = layer(4, 64, 32)
    e = torch.empty(0, 2, device="cuda")
    assert lb.mx4_moe_few(torch.empty(0, 64, device="cuda"), e.int(), e, ex).shape == (0, 64)
    ids, w = routing(65, 2, 4)
    with pytest.raises(lx.LorexError):
        lb.mx4_moe_few(tokens(65, 64, "f32"), ids, w, ex)
    ids, w, x = ids[:3].contiguous(), w[:3].contiguous(), tokens(3, 64, "f32")
    for bad in (lambda: lb.mx4_moe_few(x[:, :32].contiguous(), ids, w, ex), lambda: lb.mx4_moe_few(x, ids.long(), w, ex),
                lambda: lb.mx4_moe_few(x, ids, w[:2], ex), lambda: lb.mx4_moe_few(x.t().contiguous().t(), ids, w, ex),
                lambda: lb.mx4_moe_few(x, ids.cpu(), w, ex), lambda: lb.mx4_moe_few(x.half(), ids, w, ex),
                lambda: lb.mx4_moe_few(x, ids, w, ex, out_dtype=torch.float16)):
        with pytest.raises(ValueError):
            bad()


def test_more_workgroups_than_one_dimension_holds():
    """256 slots times rows of 2^20: 2^32 threads in the first launch. One slot names an
    expert; the weights of the others, which nothing reads, are not there."""
    require_gpu()
    T, k, E, d, f = 8, 32, 8192, 8, 1 << 20
    g = torch.Generator(device="cuda")
    g.manual_seed(3)
    u8 = lambda *s, lo, hi: torch.randint(lo, hi, s, device="cuda", generator=g, dtype=torch.uint8)  # noqa: E731
    gu = lb.Mx4(u8(2 * f, 64, lo=0, hi=255), u8(2 * f, 4, lo=124, hi=127), d)
    dn = lb.Mx4(u8(d, f // 2, lo=0, hi=255), u8(d, f // 32, lo=118, hi=121), f)
    gu.codes[:, d // 2:] = 0
    x = tokens(T, d, "f32")
    ids, w = torch.full((T, k), -1, dtype=torch.int32, device="cuda"), torch.ones(T, k, device="cuda")
    ids[5, 9], w[5, 9] = 0, 0.75
    L = lb.lib()
    n = L.lx_mx4_moe_few_workspace_bytes(T, k, E, d, f)
    ws, out = torch.empty(n, dtype=torch.uint8, device="cuda"), torch.empty(T, d, device="cuda")
    st = L.lx_mx4_moe_few(x.data_ptr(), lx.LX_F32, T, d, ids.data_ptr(), w.data_ptr(), k, E, f, gu.codes.data_ptr(), gu.scales.data_ptr(),
                          dn.codes.data_ptr(), dn.scales.data_ptr(), out.data_ptr(), lx.LX_F32, ws.data_ptr(), n,
                          torch.cuda.current_stream().cuda_stream)
    torch.cuda.synchronize()
    assert st == lx.LX_OK, L.lx_last_error()
    one = [torch.tensor([[0]], dtype=torch.int32), torch.tensor([[0.75]])]
    ex = lb.Mx4Experts(*(lb.Mx4(q.codes[None], q.scales[None], q.K) for q in (gu, dn)))
    ref, tol = reference(x[5:6], *one, ex, torch.float32)
    assert (np.abs(host(out[5:6]) - ref) <= tol).all() and not out[[0, 1, 2, 3, 4, 6, 7]].any()

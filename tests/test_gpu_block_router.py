"""The router's logits as the 4-bit block and the balance loss take them."""
import numpy as np
import pytest
import torch

from oracle import block as O
from oracle import router as R
from paper_2608_07814_amd import block as lb
from paper_2608_07814_amd import lorex as lx
from gpu_util import require_gpu, say

pytestmark = pytest.mark.gpu


def chosen(logits, k):
    """The k largest of each row, equal ones by their index."""
    return np.argsort(-logits, 1, kind="stable")[:, :k]


# few tokens split the sums over d, many do not
@pytest.mark.parametrize("T,E,d,f,k", [(1, 16, 256, 64, 2), (5, 64, 2048, 128, 8), (700, 128, 1024, 64, 8), (3000, 32, 128, 128, 2)])
def test_block_balances_the_logits_that_it_routes_by(T, E, d, f, k):
    """Ids and weights follow from the block's logits exactly, near ties as well
    (router rows that differ by little); the loss is theirs. Weights are exponentials
    and a sum of k in fp32: within 2^-18."""
    require_gpu()
    say(f"mx4_moe_block's logits T={T} E={E} d={d} k={k}")
    g = torch.Generator(device="cuda")
    g.manual_seed(T)
    r = lambda *s: torch.randn(*s, device="cuda", generator=g)  # noqa: E731
    ex = lb.mx4_experts((r(E, f, d) * d ** -0.5).bfloat16(), (r(E, f, d) * d ** -0.5).bfloat16(), (r(E, d, f) * d ** -0.5).bfloat16())
    w_r = r(E, d)
    w_r[1::2] = w_r[::2] + 0.004 * r(E // 2, d)
    out = lb.mx4_moe_block(r(T, d).bfloat16(), torch.ones(d, device="cuda").bfloat16(), w_r.bfloat16(), ex, k, balance_coef=0.5)
    torch.cuda.synchronize()
    assert out.logits.shape == (T, E) and out.logits.dtype == torch.float32
    z = out.logits.double().cpu().numpy()
    ids = out.topk_ids.cpu().numpy()
    assert np.array_equal(ids, chosen(z, k))
    top = np.take_along_axis(z, ids, 1).astype(np.float32)
    w = np.exp((top - top[:, :1]).astype(np.float64))  # (the difference of two fp32 logits is one in fp32)
    assert np.max(np.abs(out.topk_weights.double().cpu().numpy() / (w / w.sum(1, keepdims=True)) - 1)) <= 2.0 ** -18
    loss, counts, _, n, _, _ = O.balance(z, ids, None, 0.5)
    assert np.array_equal(out.balance.counts.cpu().numpy(), counts) and out.balance.n_tokens.item() == n == T
    assert abs(out.balance.loss.item() - loss) <= 4 * 256 * 2.0 ** -24 * loss


@pytest.mark.parametrize("T,d,E,k", [(1, 2048, 128, 8), (64, 2048, 128, 8), (100, 256, 8, 2), (4096, 512, 128, 8), (33, 4096, 256, 8),
                                     (50, 128, 512, 32), (7, 512, 40, 32), (5, 1216, 100, 6)])
def test_router_with_its_logits(T, d, E, k):
    """Ids and weights are lx_route_topk's bit for bit; the logits lie within the fp32
    summation bound of fp64."""
    require_gpu()
    say(f"route_topk_logits T={T} d={d} E={E} k={k}")
    g = torch.Generator(device="cuda")
    g.manual_seed(T + E)
    x, w = (torch.randn(*s, device="cuda", generator=g).bfloat16() for s in ((T, d), (E, d)))
    ids, weights, logits = lb.route_topk_logits(x, w, k)
    ref = lx.route_topk(x, w, k)
    assert torch.equal(ids, ref[0]) and torch.equal(weights, ref[1])
    bits = lambda t: t.cpu().view(torch.int16).numpy().view(np.uint16)  # noqa: E731
    assert np.all(np.abs(logits.double().cpu().numpy() - R.router_logits(bits(x), bits(w), "bf16")) <= R.fp32_sum_bound(bits(x), bits(w), "bf16"))
    assert np.array_equal(ids.cpu().numpy(), chosen(logits.cpu().numpy(), k))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            again = lb.route_topk_logits(x, w, k)
    for _ in range(3):
        for v in again:
            v.fill_(7)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(again, (ids, weights, logits)))


def test_router_with_its_logits_refuses():
    require_gpu()
    r = lambda *s: torch.randn(*s, device="cuda").bfloat16()  # noqa: E731
    for x, w in ((r(3, 128), r(8, 64)), (r(3, 128).float(), r(8, 128)), (r(3, 128), r(8, 128).float()), (r(128, 3).t(), r(8, 128)),
                 (r(3, 128), r(8, 128).cpu()), (r(128), r(8, 128))):
        with pytest.raises(ValueError):
            lb.route_topk_logits(x, w, 2)
    for d, E, k in ((128, 6, 2), (96, 8, 2), (128, 8, 9), (128, 516, 2)):
        with pytest.raises(lx.LorexError):
            lb.route_topk_logits(r(3, d), r(E, d), k)

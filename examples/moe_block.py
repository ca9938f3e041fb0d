"""A MoE block with its experts in 4 bits: a prompt, then single tokens from a HIP
graph, then the gradients of a training step around the experts.

    python examples/moe_block.py [--experts 128 --d 2048 --f 768 --k 8 --tokens 4096 --activations mx8]

Random weights with the distributions of the library's synthetic layers.
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2608_07814_amd import block as lb  # noqa: E402


def timed(f, n=20):
    for _ in range(3):
        f()
    a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    a.record()
    for _ in range(n):
        f()
    b.record()
    b.synchronize()
    return a.elapsed_time(b) / n * 1e3


def main():
    p = argparse.ArgumentParser()
    for name, v in (("experts", 128), ("d", 2048), ("f", 768), ("k", 8), ("tokens", 4096), ("decode", 16)):
        p.add_argument("--" + name, type=int, default=v)
    p.add_argument("--activations", choices=("mx4", "mx8"), default="mx4", help="of the prompt")
    p.add_argument("--decode-activations", choices=("mx4", "mx8", "full"), default="mx4", help="of the single tokens")
    p.add_argument("--dropout", type=float, default=0.0, help="of the experts' sum, in the training step")
    a = p.parse_args()
    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    r = lambda *s: torch.randn(*s, device="cuda", generator=g)  # noqa: E731
    E, d, f = a.experts, a.d, a.f
    w = [(r(E, *s) * d ** -0.5).bfloat16() for s in ((f, d), (f, d), (d, f))]
    experts = lb.mx4_experts(*w)
    del w
    w_r, w_pre, w_post, w_next = r(E, d).bfloat16(), *(1 + 0.1 * r(3, d)).bfloat16()
    block = lambda h, activations=a.activations: lb.mx4_moe_block(  # noqa: E731
        h, w_pre, w_r, experts, a.k, w_post=w_post, w_next=w_next, balance_coef=0.01, activations=activations)

    h = r(a.tokens, d).bfloat16()
    out = block(h)
    us = timed(lambda: block(h))
    print(f"prompt: {a.tokens} tokens in {us:.0f} us; balance loss {out.balance.loss.item():.5f}, "
          f"busiest expert {out.balance.counts.max().item()} of {a.tokens * a.k} slots")

    hd = r(a.decode, d).bfloat16()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())  # (the current stream makes hd)
    with torch.cuda.stream(side):
        for _ in range(2):
            eager = block(hd, a.decode_activations)
        side.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            replayed = block(hd, a.decode_activations)
    torch.cuda.current_stream().wait_stream(side)
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(replayed.h_out, eager.h_out) and torch.equal(replayed.x_next, eager.x_next)
    print(f"decode: {a.decode} tokens in {timed(graph.replay):.0f} us, replayed from a graph")

    # a training step around the experts: from the gradients of the stream and of
    # the next block's input to those of the stream, the experts' sum, the norms and
    # the router
    y = r(a.tokens, d).bfloat16()  # the experts' sum, as a training forward keeps it
    norms = dict(w_pre=w_next, w_post=w_post)
    if a.dropout:
        rng = torch.tensor([1234, 0], device="cuda")  # the generator's seed, and an offset that each step moves on
        h_out, x_next = lb.block_norm_dropout(h, y, a.dropout, rng, **norms)
    else:
        h_out, x_next = lb.block_norm(h, y, **norms)
    w_r32, x32 = w_r.float(), out.x.float()  # (the router's gradients are formed in fp32, as its logits are)
    dh_out, dx_next = r(a.tokens, d).bfloat16(), r(a.tokens, d).bfloat16()

    def step():
        if a.dropout:
            after = lb.block_norm_dropout_backward(h_out, y, dx_next, dh_out, a.dropout, rng, **norms)
        else:
            after = lb.block_norm_backward(h_out, y, dx_next, dh_out, **norms)
        dlogits = lb.balance_loss_backward(out.logits, out.balance.counts, out.balance.n_tokens, a.k, coef=0.01)
        dx = dlogits @ w_r32  # (the experts' own gradient would be added here)
        before = lb.block_norm_backward(h, None, dx, after.dh, w_pre=w_pre)
        return before.dh, after, before, dlogits.t() @ x32

    dh, after, before, dw_r = step()
    print(f"training: gradients of stream, norms and router in {timed(step):.0f} us; |dh| {dh.float().norm().item():.1f}, "
          f"|dw_r| {dw_r.float().norm().item():.2e}, |dw_post| {after.dw_post.norm().item():.1f}")


if __name__ == "__main__":
    main()

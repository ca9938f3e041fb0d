"""Calls on a stream of their own while the caller's stream is busy."""
import pytest
import torch

from paper_2608_07814_amd import block as lb
from gpu_util import require_gpu, say

pytestmark = pytest.mark.gpu


def test_experts_rounded_on_another_stream():
    """The weights are ready on the side stream, the caller's stream is busy for
    some milliseconds: the result is that of the default stream."""
    require_gpu()
    E, d, f = 8, 1024, 768
    side = torch.cuda.Stream()
    g = torch.Generator(device="cuda")
    g.manual_seed(3)
    w = [torch.randn(E, *s, device="cuda", generator=g).bfloat16() for s in ((f, d), (f, d), (d, f))]
    w[2] = w[2].transpose(1, 2).contiguous().transpose(1, 2)  # (not contiguous)
    ref = lb.mx4_experts(*w)
    torch.cuda.synchronize()
    busy = torch.randn(4096, 4096, device="cuda")
    for _ in range(20):
        busy = busy @ busy * 1e-3
    got = lb.mx4_experts(*w, side)
    side.synchronize()
    for a, b in zip((*got.gate_up[:2], *got.down[:2]), (*ref.gate_up[:2], *ref.down[:2])):
        assert torch.equal(a, b)


def test_calls_leave_memory_of_pending_work_alone():
    """The caller's stream frees blocks of the outputs' and workspace's sizes that
    its pending work still reads; a call on another stream writes elsewhere."""
    require_gpu()
    M, N, K = 64, 4096, 14336
    say(f"mx4_gemm on a side stream {M} x {N} x {K}")
    g = torch.Generator(device="cuda")
    g.manual_seed(4)
    a = lb.mx4_quantize(torch.randn(M, K, device="cuda", generator=g))
    b = lb.mx4_quantize(torch.randn(N, K, device="cuda", generator=g))
    need = lb.lib().lx_mx4_gemm_workspace_bytes(M, N, K, 1)
    assert need > 0
    ref = lb.mx4_gemm(a, b)
    side = torch.cuda.Stream()
    busy = torch.randn(4096, 4096, device="cuda", generator=g)
    torch.cuda.synchronize()
    for _ in range(20):
        busy = busy @ busy * 1e-3
    blocks = [torch.full((n,), 3, dtype=torch.uint8, device="cuda") for n in (need, M * N * 4)]
    copies = [t.clone() for t in blocks]  # (pending, like the fills that they read)
    del blocks
    got = lb.mx4_gemm(a, b, stream=side)
    side.synchronize()
    assert torch.equal(got, ref)
    torch.cuda.synchronize()
    assert all(bool((t == 3).all()) for t in copies)


def test_outputs_are_not_reused_before_the_callers_stream_is_done():
    """An output that the caller's stream still reads when it is dropped is not given
    to the call's stream's next allocation."""
    require_gpu()
    side = torch.cuda.Stream()
    x, z = torch.randn(1 << 14, 1024, device="cuda"), torch.zeros(1 << 14, 1024, device="cuda")
    busy = torch.randn(4096, 4096, device="cuda")
    torch.cuda.synchronize()
    q = lb.mx4_quantize(x, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    for _ in range(20):
        busy = busy @ busy * 1e-3
    place, codes = q.codes.data_ptr(), q.codes.clone()  # (pending)
    del q
    again = lb.mx4_quantize(z, stream=side)
    assert again.codes.data_ptr() != place
    torch.cuda.synchronize()
    assert torch.equal(codes, lb.mx4_quantize(x).codes)

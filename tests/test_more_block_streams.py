"""On which GPU, in which streams and from which memory the bindings for few tokens,
8-bit values and dropout issue their work, on the CPU, with the stand-ins of the other
bindings' test."""
import pytest

from paper_2608_07814_amd import block as lb
from paper_2608_07814_amd import lorex as lx
from test_block_streams import BF16, F32, I32, U8, Stream, Tensor, tensors, world  # noqa: F401

import torch


def calls(world, gpu):  # noqa: F811
    t = lambda dtype, *shape: Tensor(world, shape, dtype, gpu)  # noqa: E731
    h, y, w, rng = t(BF16, 4, 64), t(F32, 4, 64), t(BF16, 64), t(torch.int64, 2)
    a, b = lb.Mx8(t(U8, 4, 128), t(U8, 4, 4), 128), lb.Mx4(t(U8, 8, 64), t(U8, 8, 4), 128)
    ex = lb.Mx4Experts(lb.Mx4(t(U8, 8, 80, 64), t(U8, 8, 80, 4), 64), lb.Mx4(t(U8, 8, 64, 64), t(U8, 8, 64, 4), 40))
    return {
        "block_norm_mx8": lambda **kw: lb.block_norm_mx8(h, y, w_pre=w, w_post=w, **kw),
        "block_norm_mx8 alone": lambda **kw: lb.block_norm_mx8(h=h, w_pre=w, **kw),
        "block_norm_dropout": lambda **kw: lb.block_norm_dropout(h, y, 0.1, rng, w_pre=w, w_post=w, **kw),
        "block_norm_dropout_backward": lambda **kw: lb.block_norm_dropout_backward(h, y, h, h, 0.1, rng, w_pre=w, w_post=w, gate=t(F32, 4), **kw),
        "mx8_quantize": lambda **kw: lb.mx8_quantize(h, **kw),
        "mx8_dequantize": lambda **kw: lb.mx8_dequantize(a, **kw),
        "mx8_gemm": lambda **kw: lb.mx8_gemm(a, b, bias=t(F32, 1, 8), residual=t(BF16, 4, 8), **kw),
        "mx8_gemm into 8 bits": lambda **kw: lb.mx8_gemm(a, b, act=lb.ACT_SILU, out_dtype="mx8", **kw),
        "mx4_moe_few": lambda **kw: lb.mx4_moe_few(h, t(I32, 4, 2), t(F32, 4, 2), ex, **kw),
    }


ENTRIES = sorted(calls(None, 0))


@pytest.mark.parametrize("entry", ENTRIES)
def test_the_tensors_gpu_is_current_during_the_launch(world, entry):  # noqa: F811
    calls(world, 1)[entry]()
    ((_, device, handle, _),) = world.calls
    assert (device, handle) == (1, 0) and world.device == 0
    side = Stream(1, 77)
    calls(world, 1)[entry](stream=side)
    assert world.calls[1][1:3] == (1, 77) and world.device == 0 and world.current[1].cuda_stream == 0
    with world.on_device(1):
        calls(world, 0)[entry]()
    assert world.calls[2][1:3] == (0, 0)


@pytest.mark.parametrize("entry", ENTRIES)
def test_a_stream_of_another_gpu_is_refused(world, entry):  # noqa: F811
    with pytest.raises(ValueError):
        calls(world, 0)[entry](stream=Stream(1, 77))
    assert not world.calls


@pytest.mark.parametrize("entry", ENTRIES)
def test_memory_of_a_call_is_in_its_streams_order(world, entry):  # noqa: F811
    side, caller = Stream(0, 77), world.current[0]
    out = tensors(calls(world, 0)[entry](stream=side))
    ((_, _, handle, used),) = world.calls
    assert handle == 77 and world.made and all(t.pool == side for t in world.made)
    new = [t for t in out if t.pool is not None]
    assert new and all(caller in t.recorded for t in new)
    assert {id(t) for t in used if t.pool is not None} >= {id(t) for t in new}
    world.made.clear()
    calls(world, 0)[entry]()
    assert world.made and all(t.pool == caller for t in world.made)


INPUTS = {"block_norm_mx8": 3, "block_norm_mx8 alone": 2, "block_norm_dropout": 4, "block_norm_dropout_backward": 4, "mx8_dequantize": 2,
          "mx8_gemm": 4, "mx8_gemm into 8 bits": 4, "mx4_moe_few": 5}


@pytest.mark.parametrize("entry", sorted(INPUTS))
def test_tensors_of_two_gpus_are_refused(world, monkeypatch, entry):  # noqa: F811
    """Whichever of a call's inputs (those that are made before it) is on another GPU."""
    plain, made = Tensor.__init__, []

    def init(self, *a, **kw):
        plain(self, *a, **kw)
        made.append(self)

    monkeypatch.setattr(Tensor, "__init__", init)
    calls(world, 0)
    refused = 0
    for i in range(len(made)):
        made.clear()
        call = calls(world, 0)[entry]
        made[i].gpu = 1
        try:
            call()
        except ValueError:
            refused += 1
            assert not world.calls
        world.calls.clear()
    assert refused == INPUTS[entry]


@pytest.mark.parametrize("activations,kernels", [("mx8", 5), ("full", 3)])
def test_moe_block_runs_on_its_gpu(world, activations, kernels):  # noqa: F811
    t = lambda dtype, *shape: Tensor(world, shape, dtype, 1)  # noqa: E731
    E, d, f, k = 8, 128, 128, 2
    ex = lb.Mx4Experts(lb.Mx4(t(U8, E, 2 * f, 64), t(U8, E, 2 * f, 4), d), lb.Mx4(t(U8, E, d, 64), t(U8, E, d, 4), f))
    with pytest.MonkeyPatch.context() as m:
        m.setattr(lx, "route_topk", lambda x, w_r, k, **kw: (x.new_empty((4, k), dtype=I32), x.new_empty((4, k), dtype=F32)))
        out = lb.mx4_moe_block(t(BF16, 4, d), t(BF16, d), t(BF16, E, d), ex, k, activations=activations)
    assert {c[1] for c in world.calls} == {1} and world.device == 0 and out.h_out.gpu == 1
    assert len(world.calls) == kernels

"""On which GPU, in which streams and from which memory the bindings around the
expert layer issue their work, on the CPU: tensors, streams and the library are
stand-ins that record what happens."""
import contextlib
import ctypes
import os

import pytest
import torch

from paper_2608_07814_amd import block as lb
from paper_2608_07814_amd import lorex as lx


class Stream:
    def __init__(self, gpu, handle):
        self.device_index, self.cuda_stream = gpu, handle
        self.stream_id, self.device_type = handle, 1

    def __eq__(self, other):
        return (self.device_index, self.cuda_stream) == (other.device_index, other.cuda_stream)


class Tensor:
    """`pool` is the stream whose memory it is in, `ready` the one whose work
    fills it, `recorded` the streams whose work its release waits for."""

    def __init__(self, world, shape, dtype, gpu, pool=None):
        self.world, self.shape, self.dtype, self.gpu = world, torch.Size(shape), dtype, gpu
        self.pool, self.ready, self.recorded = pool, pool, []

    device = property(lambda self: f"cuda:{self.gpu}")

    def dim(self):
        return len(self.shape)

    def numel(self):
        return self.shape.numel()

    def get_device(self):
        return self.gpu

    def is_contiguous(self):
        return True

    def contiguous(self):
        return self

    def data_ptr(self):
        self.world.tensors[id(self)] = self
        return id(self) * 256

    def record_stream(self, stream):
        self.recorded.append(stream)

    def new_empty(self, shape, dtype=None):
        shape = (shape,) if isinstance(shape, int) else shape
        t = Tensor(self.world, shape, dtype or self.dtype, self.gpu, self.world.stream(self.gpu))
        self.world.made.append(t)
        return t

    def unbind(self, dim):
        rows = [Tensor(self.world, self.shape[1:], self.dtype, self.gpu, self.pool) for _ in range(self.shape[0])]
        for r in rows:
            r.recorded = self.recorded  # one allocation
        return rows


class World:
    """Two GPUs, each with its default stream (handle 0) and others."""

    def __init__(self):
        self.device, self.current = 0, [Stream(0, 0), Stream(1, 0)]
        self.tensors, self.made, self.calls = {}, [], []

    def stream(self, gpu=None):
        return self.current[self.device if gpu is None else gpu]

    @contextlib.contextmanager
    def on_device(self, gpu):
        before, self.device = self.device, gpu
        yield
        self.device = before

    def set_stream(self, stream_id, device_index, device_type):
        self.device = device_index
        self.current[device_index] = Stream(device_index, stream_id)

    def __getattr__(self, name):  # the library
        if not name.startswith("lx_"):
            raise AttributeError(name)
        if name.endswith("_bytes"):
            return lambda *a: 4096

        def call(*a):
            handle = a[-1] or 0
            # a handle of 0 is the default stream of the current GPU
            self.calls.append((name, self.device, handle, [self.tensors[p // 256] for p in a if isinstance(p, int) and p // 256 in self.tensors]))
            return 0
        return call


@pytest.fixture
def world(monkeypatch):
    w = World()
    monkeypatch.setattr(lb, "lib", lambda: w)
    monkeypatch.setattr(lx, "lib", lambda: w)
    monkeypatch.setattr(torch.cuda, "device", w.on_device)
    monkeypatch.setattr(torch, "Stream", lambda stream_id, device_index, device_type: Stream(device_index, stream_id))
    monkeypatch.setattr(lb, "_current_stream", lambda gpu: (w.stream(gpu).stream_id, gpu, 1))
    monkeypatch.setattr(lb, "_set_stream", w.set_stream)
    monkeypatch.setattr(lb, "_current_raw_stream", lambda gpu: w.stream(gpu).cuda_stream)
    monkeypatch.setattr(lb, "_current_device", lambda: w.device, raising=False)
    return w


def _library():
    """The library itself, for sizes (no call of it reaches a launch)."""
    if not os.path.exists(lx.LIB_PATH):
        from paper_2608_07814_amd import build
        build.build()
    L = ctypes.CDLL(lx.LIB_PATH)
    fn = L.lx_moe_tree_workspace_bytes
    fn.restype, fn.argtypes = lx.EXPORTS["lx_moe_tree_workspace_bytes"]
    return L


F32, BF16, I32, U8 = torch.float32, torch.bfloat16, torch.int32, torch.uint8


def calls(world, gpu):
    """Every entry that takes a stream, on tensors of one GPU."""
    t = lambda dtype, *shape: Tensor(world, shape, dtype, gpu)  # noqa: E731
    h, y, w = t(BF16, 4, 64), t(F32, 4, 64), t(BF16, 64)
    a, b = lb.Mx4(t(U8, 4, 64), t(U8, 4, 4), 128), lb.Mx4(t(U8, 8, 64), t(U8, 8, 4), 128)
    return {
        "block_norm": lambda **kw: lb.block_norm(h, y, w_pre=w, w_post=w, **kw),
        "block_norm by names": lambda **kw: lb.block_norm(h=h, w_pre=w, **kw),
        "block_norm_backward": lambda **kw: lb.block_norm_backward(h, y, h, h, w_pre=w, w_post=w, gate=t(F32, 4), **kw),
        "route_topk_logits": lambda **kw: lb.route_topk_logits(h, t(BF16, 8, 64), 2, **kw),
        "balance_loss": lambda **kw: lb.balance_loss(h, t(I32, 4, 2), **kw),
        "balance_loss_backward": lambda **kw: lb.balance_loss_backward(h, t(I32, 64), t(I32, 1), 2, **kw),
        "mx4_quantize": lambda **kw: lb.mx4_quantize(h, **kw),
        "mx4_dequantize": lambda **kw: lb.mx4_dequantize(a, **kw),
        "mx4_gemm": lambda **kw: lb.mx4_gemm(a, b, **kw),
    }


ENTRIES = sorted(calls(None, 0))


@pytest.mark.parametrize("entry", ENTRIES)
def test_the_tensors_gpu_is_current_during_the_launch(world, entry):
    """A launch on stream 0, and any without a stream, goes to the current GPU."""
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
def test_a_stream_of_another_gpu_is_refused(world, entry):
    with pytest.raises(ValueError):
        calls(world, 0)[entry](stream=Stream(1, 77))
    assert not world.calls


def test_moe_block_runs_on_its_gpu(world):
    t = lambda dtype, *shape: Tensor(world, shape, dtype, 1)  # noqa: E731
    E, d, f, k = 8, 128, 128, 2
    ex = lb.Mx4Experts(lb.Mx4(t(U8, E, 2 * f, 64), t(U8, E, 2 * f, 4), d), lb.Mx4(t(U8, E, d, 64), t(U8, E, d, 4), f))
    with pytest.MonkeyPatch.context() as m:
        m.setattr(lx, "route_topk", lambda x, w_r, k, **kw: (x.new_empty((4, k), dtype=I32), x.new_empty((4, k), dtype=F32)))
        out = lb.mx4_moe_block(t(BF16, 4, d), t(BF16, d), t(BF16, E, d), ex, k)
    assert len(world.calls) == 7 and {c[1] for c in world.calls} == {1} and world.device == 0
    assert out.h_out.gpu == 1


def tensors(r):
    return [t for v in r for t in tensors(v)] if isinstance(r, tuple) else [r] if isinstance(r, Tensor) else []


@pytest.mark.parametrize("entry", ENTRIES)
def test_memory_of_a_call_is_in_its_streams_order(world, entry):
    """What a call allocates, workspaces among it, is memory of the call's stream:
    memory of another stream's pool may still be in use by that stream's pending
    work. What is handed to the caller is not reused before the caller's stream,
    as it stood at the call, is done with it."""
    side, caller = Stream(0, 77), world.current[0]
    out = tensors(calls(world, 0)[entry](stream=side))
    ((_, _, handle, used),) = world.calls
    assert handle == 77 and world.made
    for t in world.made:
        assert t.pool == side
    new = [t for t in out if t.pool is not None]
    assert new and all(caller in t.recorded for t in new)
    assert {id(t) for t in used if t.pool is not None} >= {id(t) for t in new}
    world.made.clear()
    calls(world, 0)[entry]()
    assert world.made and all(t.pool == caller for t in world.made)


def test_experts_are_rounded_in_one_stream(world, monkeypatch):
    """Joining the projections, making them contiguous, rounding: all of it in the
    given stream (else the rounding may read what is not yet written), the
    temporaries in its memory."""
    side, caller, where = Stream(0, 77), world.current[0], []

    def cat(parts, dim):
        where.append(world.stream())
        return parts[0].new_empty((8, 256, 128))

    def contiguous(self):
        where.append(world.stream())
        return self.new_empty(self.shape)

    monkeypatch.setattr(torch, "cat", cat)
    monkeypatch.setattr(Tensor, "contiguous", contiguous)
    w = Tensor(world, (8, 128, 128), BF16, 0)
    for give in (lambda: lb.mx4_experts(w, w, w, side), lambda: lb.mx4_experts(w, w, w, stream=side)):
        ex = give()
        assert len(where) >= 2 and all(s == side for s in where)
        assert [c[2] for c in world.calls] == [77, 77] and all(t.pool == side for t in world.made)
        assert all(caller in t.recorded for t in tensors(ex)) and len(tensors(ex)) == 4
        for v in (where, world.calls, world.made):
            v.clear()
    lb.mx4_experts(w, w, w)
    assert all(s == caller for s in where) and [c[2] for c in world.calls] == [0, 0]
    where.clear()
    w.gpu = 1
    lb.mx4_experts(w, w, w)
    assert {c[1] for c in world.calls[2:]} == {1} and all(s == world.current[1] for s in where)
    with pytest.raises(ValueError):
        lb.mx4_experts(w, w, w, side)


@pytest.mark.parametrize("T,E,d,f,k", [(4096, 128, 2048, 768, 8), (8192, 8, 4096, 14336, 2)])
def test_moe_block_reserves_what_bucketing_needs(world, monkeypatch, T, E, d, f, k):
    """The block's workspace follows the slots, not the experts' sizes: a forward of
    these layers would take up to 2.9 GiB."""
    real = _library()
    monkeypatch.setattr(World, "lx_moe_tree_workspace_bytes", lambda self, *a: real.lx_moe_tree_workspace_bytes(*a), raising=False)
    monkeypatch.setattr(lx, "route_topk", lambda x, w_r, k, **kw: (x.new_empty((T, k), dtype=I32), x.new_empty((T, k), dtype=F32)))
    t = lambda dtype, *shape: Tensor(world, shape, dtype, 0)  # noqa: E731
    q = lambda *s: lb.Mx4(t(U8, *s[:-1], lb.mx4_padded(s[-1]) // 2), t(U8, *s[:-1], lb.mx4_padded(s[-1]) // 32), s[-1])  # noqa: E731
    ex = lb.Mx4Experts(q(E, 2 * f, d), q(E, d, f))
    lb.mx4_moe_block(t(BF16, T, d), t(BF16, d), t(BF16, E, d), ex, k)
    (ws,) = [m for m in world.made if m.dtype == U8 and m.dim() == 1 and m.numel() != 4096]
    assert ws.numel() <= 1200 * T * k + (8 << 20)

"""The order of the streams in examples/moe_block.py, on the CPU: a stand-in for
torch notes for every value which stream makes it, and for every use whether that
stream's work so far comes before it."""
import contextlib
import importlib.util
import os
from types import SimpleNamespace

import torch


class Stream:
    def __init__(self, world):
        self.world, self.before = world, set()

    def wait_stream(self, other):
        self.before |= other.before

    def synchronize(self):
        self.world.host |= self.before


class World:
    def __init__(self):
        self.host, self.count, self.late = set(), 0, []
        self.default = self.current = Stream(self)
        self.streams = [self.default]
        self.captured = None

    def op(self, deps, what):
        s = self.current
        s.before |= self.host
        self.late += [what for v in deps if isinstance(v, Value) and v.op not in s.before]
        self.count += 1
        s.before.add(self.count)
        return self.count

    def wait_for_all(self):
        for s in self.streams:
            s.synchronize()

    def new_stream(self):
        self.streams.append(Stream(self))
        return self.streams[-1]

    @contextlib.contextmanager
    def on(self, s):
        before, self.current = self.current, s
        yield
        self.current = before

    @contextlib.contextmanager
    def graph(self, g, stream):
        self.wait_for_all()
        with self.on(stream):
            g.values = self.captured = []
            yield
            self.captured = None


class Value:
    def __init__(self, world, deps=(), what=""):
        self.world, self.op = world, world.op(deps, what)
        if world.captured is not None:
            world.captured.append(self)

    def make(self, what, *deps):
        return Value(self.world, (self, *deps), what)

    def __iter__(self):
        return (self.make("row") for _ in range(3))

    def __getattr__(self, name):
        return lambda *a, **kw: self.make(name, *a)

    def item(self):
        self.make("item")
        self.world.current.synchronize()
        return 1.0

    def __add__(self, o):
        return self.make("sum", o)

    __radd__ = __mul__ = __rmul__ = __matmul__ = __add__


class Graph:
    def __init__(self, world):
        self.world = world

    def replay(self):
        op = self.world.op((), "replay")
        for v in self.values:
            v.op = op


def test_streams_wait_for_what_they_use(root, monkeypatch):
    spec = importlib.util.spec_from_file_location("moe_block_example", os.path.join(root, "examples", "moe_block.py"))
    ex = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(ex)
    w = World()
    event = SimpleNamespace(record=lambda: None, synchronize=lambda: w.current.synchronize(), elapsed_time=lambda o: 1.0)
    cuda = SimpleNamespace(Stream=w.new_stream, stream=w.on, current_stream=lambda: w.current, synchronize=w.wait_for_all,
                           CUDAGraph=lambda: Graph(w), graph=lambda g, stream: w.graph(g, stream), Event=lambda **kw: event)

    class Torch:
        randn = staticmethod(lambda *s, **kw: Value(w))
        Generator = staticmethod(lambda **kw: SimpleNamespace(manual_seed=lambda n: None))

        def __getattr__(self, name):
            return getattr(torch, name)

    def equal(a, b):
        a.make("equal", b).item()
        return True

    fake = Torch()
    fake.cuda, fake.equal = cuda, equal
    v = lambda *deps: Value(w, deps, "library")  # noqa: E731

    def moe_block(h, *a, **kw):
        out = v(h, *[x for x in (*a, *kw.values()) if isinstance(x, Value)])
        balance = SimpleNamespace(loss=v(out), counts=v(out), n_tokens=v(out))
        return SimpleNamespace(h_out=v(out), x_next=v(out), x=v(out), logits=v(out), balance=balance)

    def backward(*a, **kw):
        out = v(*a, *kw.values())
        return SimpleNamespace(dh=v(out), dy=v(out), dw_pre=v(out), dw_post=v(out))

    monkeypatch.setattr(ex, "torch", fake)
    monkeypatch.setattr(ex, "lb", SimpleNamespace(
        mx4_experts=lambda *a, **kw: v(*a), mx4_moe_block=moe_block, block_norm=lambda *a, **kw: (v(*a), v(*a)),
        block_norm_backward=backward, balance_loss_backward=lambda *a, **kw: v(*a)))
    monkeypatch.setattr("sys.argv", ["moe_block.py"])
    ex.main()
    assert w.count > 100 and not w.late, w.late

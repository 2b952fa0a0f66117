"""Whose memory a Context works in and for how long it keeps it, without a GPU: the library, the allocator and the streams are
stand-ins that write down what is asked of them."""
import contextlib

import pytest
import torch

import paper_1409_5705_amd as sfb
from paper_1409_5705_amd import binding


class Stream:
    def __init__(self, number):
        self.cuda_stream = self.stream_id = number


class Memory:
    """A device tensor's stand-in: its size, the stream it was allocated on, the other streams it was said to be used on."""

    def __init__(self, size, stream):
        self.size, self.stream, self.used_on = size, stream, []

    def numel(self):
        return self.size

    def element_size(self):
        return 1

    def data_ptr(self):
        return id(self)

    def record_stream(self, stream):
        self.used_on.append(stream)


class Machine:
    def __init__(self):
        self.default, self.side = Stream(1), Stream(2)
        self.current, self.captured = self.default, None
        self.bytes = {"sfb_apply_workspace_bytes": 100, "sfb_adapter_forward_workspace_bytes": 100}

    def __getattr__(self, name):          # the library: every call succeeds, every query is answered from `bytes`
        if not name.startswith("sfb_"):
            raise AttributeError(name)
        return lambda *args: self.bytes.get(name, 0)

    @contextlib.contextmanager
    def on(self, stream):
        before, self.current = self.current, stream or self.current
        yield
        self.current = before

    @contextlib.contextmanager
    def capture(self, stream):
        with self.on(stream):
            self.captured = stream
            yield
        self.captured = None


@pytest.fixture()
def machine(monkeypatch):
    m = Machine()
    monkeypatch.setattr(binding, "lib", lambda: m)
    monkeypatch.setattr(binding, "_ptr", lambda t, *args, **kw: None if t is None else id(t))
    monkeypatch.setattr(binding.Context, "_at", lambda self, t, *args: id(t))
    monkeypatch.setattr(torch, "empty", lambda size, **kw: Memory(size, m.current))
    monkeypatch.setattr(torch.cuda, "stream", m.on)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    monkeypatch.setattr(torch._C, "_cuda_getCurrentStream", lambda index: (m.current.stream_id, index, 1), raising=False)
    monkeypatch.setattr(torch._C, "_cuda_isCurrentStreamCapturing", lambda: m.current is m.captured, raising=False)
    return m


class List:
    """What a Context sees of a TensorList of many tensors."""

    def __init__(self, table):
        self.device, self.workspace_bytes, self.items, self.count = None, 10, None, 200
        self.table, self.table_ptr = table, table.data_ptr()

    def can_clip(self):
        return True


def clip(ctx, table):
    ctx.sfb_clip_grads(List(table), 1.0, torch.zeros(1))


def test_table_of_another_stream(machine):
    """The kernels read a list's table on the context's stream, whichever stream it was made on: its memory is not given to
    another list before they are through."""
    ctx = sfb.Context(0, stream=machine.side)
    table = Memory(4096, machine.default)
    clip(ctx, table)
    assert table.used_on == [machine.side]
    ctx.sfb_grad_norm(List(table), torch.zeros(1))
    assert machine.side in table.used_on


@pytest.mark.parametrize("inside", [True, False])
def test_table_of_a_captured_call(machine, inside):
    """A graph reads it again at every replay: it stays for as long as the context does, whether the context's stream or another one
    is the current one during the capture."""
    ctx = sfb.Context(0, stream=machine.side)
    table = Memory(4096, machine.side)
    other = Memory(4096, machine.side)
    with machine.capture(machine.side), contextlib.nullcontext() if inside else machine.on(machine.default):
        clip(ctx, table)
    clip(ctx, other)
    assert holds(ctx, table) and not holds(ctx, other)


def holds(ctx, memory):
    """Whether anything that the context keeps is `memory`."""
    def within(v):
        if isinstance(v, dict):
            return any(within(x) for x in v.values())
        if isinstance(v, (list, tuple, set)):
            return any(within(x) for x in v)
        return v is memory
    return within(vars(ctx))

"""Which stream the history encoder's calls take their memory for: no GPU in it.  CPU tensors, a library that notes what it is
called with, and streams that are numbers stand in for one."""
import contextlib

import pytest
import torch

import paper_2604_24073_amd as fs
from paper_2604_24073_amd import binding

CURRENT, NAMED = 0x100, 0x200


class Library:
    def __init__(self):
        self.calls = []

    def __getattr__(self, name):
        if name.endswith("_work_bytes"):
            return lambda *args: 64
        return lambda *args: self.calls.append((name, args[-1])) or 0


class Context:
    device, handle = -1, None                       # what CPU tensors say they are on

    def __init__(self):
        self.lib = Library()


@pytest.fixture
def streams(monkeypatch):
    """The current stream's handle, last; every allocation is noted with the one it is made for."""
    current, taken = [CURRENT], []

    @contextlib.contextmanager
    def switch(stream):
        current.append(stream)
        yield
        current.pop()

    def noted(make):
        def call(*args, **named):
            taken.append(current[-1])
            return make(*args, **named)
        return call

    monkeypatch.setattr(binding, "_current_raw_stream", lambda device: current[-1])
    monkeypatch.setattr(torch.cuda, "ExternalStream", lambda handle, device=None: handle)
    monkeypatch.setattr(torch.cuda, "stream", switch)
    monkeypatch.setattr(torch, "empty", noted(torch.empty))
    monkeypatch.setattr(torch, "empty_like", noted(torch.empty_like))
    return taken


def block(call):
    x, w = torch.zeros(6, 32), torch.ones(32)
    if call == "forward":
        return fs.fs_block_norm, (x, x, x, w, w, w), {"pack": ("a", "y")}
    return fs.fs_block_norm_backward, (x, x, x, x, x, w, w, w), {}


def attention(call):
    x, offs = torch.zeros(6, 2, 8), torch.tensor([0, 2, 6])
    args = (x, x, x, offs, offs, torch.zeros(3, 2), torch.zeros(5, dtype=torch.int32))
    if call == "backward":
        return fs.fs_jagged_attention_backward, (x, {"out": x, "lse": torch.zeros(2, 6)}) + args, {}
    return fs.fs_jagged_attention, args, {"keep": True, "max_q": 4 if call == "few rows" else 0}


def rows8(call):
    if call == "pack":
        return fs.fs_rows_pack8, (torch.zeros(6, 32),), {}
    return fs.fs_rows_unpack8, (fs.Rows8(torch.zeros(6, 32, dtype=torch.int8), torch.zeros(6, 1, dtype=torch.uint8)),), {}


CALLS = [(block, "forward"), (block, "backward"), (attention, "forward"), (attention, "few rows"), (attention, "backward"),
         (rows8, "pack"), (rows8, "unpack")]


@pytest.mark.parametrize("make,call", CALLS)
@pytest.mark.parametrize("stream", [None, CURRENT, NAMED])
def test_memory_is_taken_for_the_stream_of_the_call(streams, make, call, stream):
    function, args, named = make(call)
    streams.clear()
    ctx = Context()
    function(ctx, *args, **named, stream=stream)
    want = stream or CURRENT
    assert ctx.lib.calls == [(function.__name__, want)]
    assert streams and set(streams) == {want}


def test_a_stream_by_its_place(streams):
    x = torch.zeros(6, 32)
    for args in ((x, None, NAMED), (x, None)):
        streams.clear()
        ctx = Context()
        fs.fs_rows_pack8(ctx, *args)
        want = NAMED if len(args) == 3 else CURRENT
        assert ctx.lib.calls == [("fs_rows_pack8", want)] and set(streams) == {want}
    with pytest.raises(ValueError):
        fs.fs_rows_pack8(Context(), x, None, NAMED, 1)

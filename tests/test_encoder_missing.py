"""Calls of the history encoder that leave out what they need say so: no GPU in it."""
import pytest
import torch

import paper_2604_24073_amd as fs
from test_encoder_streams import Context

X, W = torch.zeros(6, 32), torch.ones(32)
HEADS, OFFSETS = torch.zeros(6, 2, 8), torch.tensor([0, 2, 6])
KEPT = {"out": HEADS, "lse": torch.zeros(2, 6)}


def attend(ctx, **changes):
    return fs.fs_jagged_attention(ctx, HEADS, HEADS, changes.pop("v", HEADS), OFFSETS, OFFSETS, **changes)


def attend_backward(ctx, dout=HEADS, kept=KEPT, **changes):
    return fs.fs_jagged_attention_backward(ctx, dout, kept, HEADS, HEADS, HEADS, OFFSETS, OFFSETS, **changes)


@pytest.mark.parametrize("what,call", [
    ("g", lambda c: fs.fs_block_norm(c, X, X, None, W, W, W)), ("w_post", lambda c: fs.fs_block_norm(c, X, X, X, None, W, W)),
    ("scale", lambda c: fs.fs_block_norm(c, X, X, X, W, None)), ("x", lambda c: fs.fs_block_norm(c, None, w_pre=W)),
    ("w_pre", lambda c: fs.fs_block_norm_backward(c, X, X, y=X)), ("y", lambda c: fs.fs_block_norm_backward(c, X, X, w_pre=W)),
    ("g", lambda c: fs.fs_block_norm_backward(c, X, None, X, None, None, W, W)),
    ("scale", lambda c: fs.fs_block_norm_backward(c, X, None, X, X, None, W)),
    ("dy, dh, a or y", lambda c: fs.fs_block_norm_backward(c, None, None)), ("rows", lambda c: fs.fs_rows_pack8(c, None)),
    ("v", lambda c: attend(c, v=None)), ("bucket_of", lambda c: attend(c, bias=torch.zeros(3, 2))),
    ("bias", lambda c: attend(c, bias=torch.zeros(0, 2), bucket_of=torch.zeros(5, dtype=torch.int32))),
    ("bias", lambda c: attend(c, bias=torch.tensor(0.0), bucket_of=torch.zeros(5, dtype=torch.int32))),
    ("bias", lambda c: attend(c, bias=torch.zeros(3), bucket_of=torch.zeros(5, dtype=torch.int32))),
    ("dout", lambda c: attend_backward(c, dout=None)), ("kept['lse']", lambda c: attend_backward(c, kept={"out": HEADS, "lse": None})),
    ("bucket_of", lambda c: attend_backward(c, bias=torch.zeros(3, 2)))])
def test_what_is_missing_is_named(what, call, monkeypatch):
    monkeypatch.setattr(fs.binding, "_current_raw_stream", lambda device: 1)
    ctx = Context()
    with pytest.raises(ValueError) as refusal:
        call(ctx)
    assert str(refusal.value).startswith(what + ":")
    assert not ctx.lib.calls


@pytest.mark.parametrize("max_q,want", [(0, 0), (3, 3), (-1, -1), ((1 << 31) - 1, (1 << 31) - 1), (1 << 31, (1 << 31) - 1),
                                        ((1 << 32) + 1, (1 << 31) - 1), (1 << 70, (1 << 31) - 1)])
def test_a_bound_of_rows_beyond_32_bits(max_q, want, monkeypatch):
    monkeypatch.setattr(fs.binding, "_current_raw_stream", lambda device: 1)
    ctx, seen = Context(), []
    ctx.lib.fs_jagged_attention = lambda handle, rec, stream: seen.append(rec.max_q) or 0
    attend(ctx, max_q=max_q)
    assert seen == [want]

"""Entries of the records that a call does not read may hold anything: here an address that is not aligned, strides and sizes that
no call would take."""
import pytest
import torch

import paper_2604_24073_amd as fs
from test_gpu_jagged_attention import BF16, F32, Case

pytestmark = pytest.mark.gpu

STRIDES = {"a_stride", "g_stride", "da_stride", "dg_stride", "dq_stride", "dk_stride", "dv_stride", "num_buckets", "num_distances",
           "work_bytes"}


class Spoilt:
    """A context whose calls find something in the entries named, all of which they have no use for."""

    def __init__(self, ctx, junk, names):
        self.real, self.device, self.handle, self.lib, self.check = ctx, ctx.device, ctx.handle, self, ctx.check
        self.junk, self.names, self.spoilt = junk, names, 0

    def __getattr__(self, call):
        real = getattr(self.real.lib, call)
        if call.endswith("_work_bytes"):
            return real

        def run(handle, rec, stream):
            for name in self.names:
                assert not getattr(rec, name) or name == "work", name
                setattr(rec, name, 7 if name in STRIDES else self.junk.data_ptr() + 2)
            self.spoilt += 1
            return real(handle, rec, stream)
        return run


@pytest.fixture(scope="module")
def ctx():
    c = fs.Context(max_ids=1024)
    yield c
    assert fs.fs_check_async(c) == fs.FS_OK, c.last_error()
    c.close()


def same_with(ctx, names, call):
    junk = torch.full((1 << 16,), 77, dtype=torch.uint8, device="cuda")
    want = call(ctx)
    spoilt = Spoilt(ctx, junk, names.split())
    got = call(spoilt)
    assert spoilt.spoilt == 1 and set(got) == set(want)
    for name in want:
        assert all(torch.equal(x, y) for x, y in zip(got[name], want[name])), name
    assert bool((junk == 77).all())


BACKWARD = "dy dh dx da dg da_stride dg_stride dw_post dscale dw_pre work work_bytes"


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_block_norm(ctx, dtype):
    gen = torch.Generator().manual_seed(0)
    rnd = lambda *s: torch.randn(s, generator=gen)  # noqa: E731
    x, a, g, dy, dh = (rnd(100, 64).to(t).cuda() for t in (F32, dtype, dtype, F32, dtype))
    w_post, scale, w_pre = (rnd(64).cuda() for _ in range(3))
    same_with(ctx, "a_exps g_exps y_exps " + BACKWARD, lambda c: fs.fs_block_norm(c, x, a, g, w_post, scale, w_pre))
    same_with(ctx, "w_pre " + BACKWARD, lambda c: fs.fs_block_norm(c, x, a, g, w_post, scale))
    same_with(ctx, "g a_stride g_stride w_post scale y a_codes g_codes a_exps g_exps " + BACKWARD,
              lambda c: fs.fs_block_norm(c, x, w_pre=w_pre, dtype=dtype))
    kept = fs.fs_block_norm(ctx, x, a, g, w_post, scale, w_pre, pack=("a", "g", "y"))
    same_with(ctx, "x h a_codes a_exps g_codes g_exps y_codes y_exps",
              lambda c: fs.fs_block_norm_backward(c, dy, dh, a, g, kept["y"], w_post, scale, w_pre))
    same_with(ctx, "x h a_stride g_stride",
              lambda c: fs.fs_block_norm_backward(c, dy, dh, kept["a8"], kept["g8"], kept["y8"], w_post, scale, w_pre))
    same_with(ctx, "x h y y_codes y_exps w_pre dw_pre a_codes g_codes",
              lambda c: fs.fs_block_norm_backward(c, dy, None, a, g, None, w_post, scale))
    same_with(ctx, "x h g g_codes a_exps g_exps a_stride g_stride w_post scale da dg da_stride dg_stride dw_post dscale y_codes",
              lambda c: fs.fs_block_norm_backward(c, dy, dh, y=x, w_pre=w_pre))


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("buckets", [0, 5])
def test_jagged_attention(ctx, dtype, buckets):
    c = Case([70, 3, 129], dtype=dtype, buckets=buckets)
    table = "" if buckets else " bucket_of num_buckets num_distances"
    unrounded = " out_f32" if dtype == F32 else ""
    backward = "dout dq dk dv dq_stride dk_stride dv_stride dbias"
    same_with(ctx, backward + " work work_bytes" + table + unrounded, lambda x: c.forward(x, keep=True))
    few = Case([3, 2], [300, 40], dtype=dtype, buckets=buckets)
    same_with(ctx, backward + table + unrounded, lambda x: few.forward(x, max_q=3))
    kept = c.forward(ctx, keep=True)
    same_with(ctx, (table + unrounded + (" dbias" if not buckets else "")).strip(), lambda x: c.backward(x, kept))

"""Attention over a jagged batch with a learned relative position bias, against its definition in 64 bits."""
import numpy as np
import pytest
import torch

import paper_2604_24073_amd as fs
from encoder_refs import assert_bounded, attention

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16


@pytest.fixture(scope="module")
def ctx():
    c = fs.Context(max_ids=1024)
    yield c
    assert fs.fs_check_async(c) == fs.FS_OK, c.last_error()
    c.close()


def offsets(lens):
    return torch.tensor(np.concatenate([[0], np.cumsum(lens)]), dtype=torch.int64)


class Case:
    """Inputs of a call, on the host; `lens_q` rows of q, `lens_k` keys in use and `rooms` rows of k for each user."""

    def __init__(self, lens_q, lens_k=None, rooms=None, heads=2, kv_heads=2, width=32, dtype=F32, causal=True, buckets=8,
                 distances=33, scale=None, seed=0):
        self.lens_q, self.lens_k = list(lens_q), list(lens_q if lens_k is None else lens_k)
        self.rooms = list(self.lens_k if rooms is None else rooms)
        self.padded = rooms is not None
        self.dtype, self.causal, self.scale = dtype, causal, scale
        gen = torch.Generator().manual_seed(seed)
        rnd = lambda *shape: torch.randn(shape, generator=gen)  # noqa: E731
        nq, nk = sum(self.lens_q), sum(self.rooms)
        self.q, self.k, self.v = rnd(nq, heads, width).to(dtype), rnd(nk, kv_heads, width).to(dtype), rnd(nk, kv_heads, width).to(dtype)
        self.dout = rnd(nq, heads, width).to(dtype)
        self.bias = self.bucket_of = None
        if buckets:
            self.bias = rnd(buckets, heads)
            size = distances if causal else 2 * distances - 1
            near = torch.randint(0, buckets, (min(size, 40),), generator=gen)      # buckets in no order, then runs of them
            runs = torch.randint(0, buckets, (size // 50 + 1,), generator=gen).repeat_interleave(50)
            self.bucket_of = torch.cat([near, runs])[:size].to(torch.int32)

    def layout(self):
        return {"q_offsets": offsets(self.lens_q).cuda(), "kv_offsets": offsets(self.rooms).cuda()}

    def options(self):
        o = {"causal": self.causal, "scale": self.scale}
        if self.bias is not None:
            o.update(bias=self.bias.cuda(), bucket_of=self.bucket_of.cuda())
        if self.padded:
            o["kv_lengths"] = torch.tensor(self.lens_k, dtype=torch.int64).cuda()
        return o

    def forward(self, ctx, **more):
        lay = self.layout()
        return fs.fs_jagged_attention(ctx, self.q.cuda(), self.k.cuda(), self.v.cuda(), lay["q_offsets"], lay["kv_offsets"],
                                      **self.options(), **more)

    def backward(self, ctx, kept, **more):
        lay = self.layout()
        return fs.fs_jagged_attention_backward(ctx, self.dout.cuda(), kept, self.q.cuda(), self.k.cuda(), self.v.cuda(),
                                               lay["q_offsets"], lay["kv_offsets"], **self.options(), **more)

    def want(self, grads=True):
        scale = self.q.shape[2] ** -0.5 if self.scale is None else self.scale
        return attention(self.q.double(), self.k.double(), self.v.double(), self.lens_q, self.lens_k, self.rooms,
                         None if self.bias is None else self.bias.double(), self.bucket_of, self.causal, scale, self.dtype,
                         self.dout.double() if grads else None)

    def check(self, ctx, grads=True, **more):
        want = self.want(grads)
        got = self.forward(ctx, keep=True, **more)
        if self.dtype == BF16:
            assert_bounded(got["out_f32"], *want["out"], "out_f32")
        for name in ("out", "lse"):
            assert_bounded(got[name], *want[name], name)
        if grads:
            back = self.backward(ctx, got)
            assert set(back) == {"dq", "dk", "dv"} | ({"dbias"} if self.bias is not None else set())
            for name in back:
                assert_bounded(back[name], *want[name], name)
        return got


EDGES = [0, 1, 2, 15, 16, 17, 63, 64, 65, 0, 127, 128, 129, 1, 200]


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("width", [8, 32, 40, 64, 96, 128])
def test_lengths_and_widths(ctx, dtype, causal, width):
    Case(EDGES, width=width, dtype=dtype, causal=causal, seed=width).check(ctx)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("heads,kv_heads", [(1, 1), (3, 3), (4, 1), (6, 2), (8, 8), (5, 1)])
def test_heads(ctx, dtype, heads, kv_heads):
    Case([5, 70, 131, 0, 33], heads=heads, kv_heads=kv_heads, width=32, dtype=dtype, seed=heads).check(ctx)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("buckets,distances", [(0, 0), (1, 1), (1, 300), (7, 2), (32, 32), (300, 300), (64, 128), (13, 1000), (1024, 4096)])
def test_bias_tables(ctx, dtype, causal, buckets, distances):
    Case([300, 64, 1, 150], buckets=buckets, distances=distances, dtype=dtype, causal=causal, seed=buckets + distances).check(ctx)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("run", [17, 50, 134])
@pytest.mark.parametrize("width", [32, 64])
def test_buckets_that_begin_anywhere_in_a_tile(ctx, dtype, causal, run, width):
    """Runs of distances that share a bucket: none, one or several begin in a tile, at every place in it.  Wavefronts of 16 and,
    with bf16 rows of 64 columns, of 32 query rows."""
    for shift in range(0, run, run // 8):
        c = Case([650 if width == 32 else 900, 130], heads=1, kv_heads=1, width=width, dtype=dtype, causal=causal, buckets=100, distances=600, seed=shift)
        c.bucket_of = ((torch.arange(c.bucket_of.shape[0]) + shift) // run).to(torch.int32)
        c.check(ctx)


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_widest_with_the_largest_tables(ctx, dtype):
    for causal in (True, False):
        Case([150, 65], width=128, heads=2, kv_heads=1, buckets=1024, distances=4096, dtype=dtype, causal=causal).check(ctx)


@pytest.mark.parametrize("width", [4, 12, 20, 100])
def test_widths_of_32_bit_rows(ctx, width):
    Case([70, 3, 129], width=width, seed=width).check(ctx)


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_long_histories(ctx, dtype):
    """Long enough for the form with 32 rows a wavefront, for tiles behind the last distance and for many turns."""
    Case([700, 1500, 3, 260], heads=2, kv_heads=1, width=64, dtype=dtype, buckets=20, distances=200).check(ctx)
    Case([900], heads=2, kv_heads=1, width=64, dtype=dtype, buckets=20, distances=100, causal=False, scale=0.3).check(ctx)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("width", [32, 48, 128])
def test_the_longer_the_histories_the_more_rows_at_a_time(ctx, dtype, causal, width):
    """Averages on either side of every rule's border, and others."""
    for lens in ([255, 256], [257, 256], [100, 157], [511, 512], [600, 424], [1100, 950]):
        c = Case(lens, heads=1, kv_heads=1, width=width, dtype=dtype, causal=causal, buckets=16, distances=150, seed=width)
        c.bucket_of = (torch.arange(c.bucket_of.shape[0]) // 19 % 16).to(torch.int32)
        c.check(ctx)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("causal", [True, False])
def test_fewer_and_more_query_rows_than_keys(ctx, dtype, causal):
    """Rows in front of the first key see nothing where nobody looks ahead; users without keys; caches with rows to spare."""
    c = Case([5, 70, 130, 64, 3, 40], [100, 70, 60, 0, 200, 7], [100, 128, 64, 64, 256, 7], dtype=dtype, causal=causal, heads=4, kv_heads=2)
    got = c.check(ctx)
    first = 5 + 70
    if causal:
        assert bool((got["out"][first:first + 70] == 0).all()) and bool((got["lse"][:, first:first + 70] == -np.inf).all())
    assert bool((got["out"][first + 130:first + 194] == 0).all())


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("rows,heads,kv_heads,width", [(1, 2, 2, 64), (1, 8, 1, 128), (4, 4, 2, 32), (16, 3, 3, 40), (3, 5, 1, 8)])
def test_few_rows_against_a_cache(ctx, dtype, causal, rows, heads, kv_heads, width):
    keys = [1, 0, 2, 64, 255, 256, 257, 600, 1, 1500, 300]
    nq = [rows] * 9 + [0, max(rows - 1, 1)]
    c = Case(nq, keys, [x + 70 for x in keys], heads=heads, kv_heads=kv_heads, width=width, dtype=dtype, causal=causal, buckets=9,
             distances=400, seed=rows)
    got = c.check(ctx, grads=False, max_q=rows)
    back, want = c.backward(ctx, got), c.want()
    for name in back:
        assert_bounded(back[name], *want[name], name)
    plain = c.forward(ctx)                               # the other form; one value in one type, two ways to it
    want = c.want(False)["out"]
    assert_bounded(plain["out"], *want, "plain")
    only = c.forward(ctx, max_q=rows)
    assert set(only) == {"out"} and torch.equal(only["out"], got["out"])


def test_one_long_cache(ctx):
    """Chunks of more than one turn, and more of them than lanes."""
    c = Case([1, 2], [200_000, 90_000], heads=16, kv_heads=8, width=32, dtype=BF16, buckets=16, distances=4096)
    c.check(ctx, grads=False, max_q=2)


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_parts_of_one_tensor(ctx, dtype):
    c = Case([70, 1, 129, 64], heads=4, kv_heads=2, width=32, dtype=dtype)
    lay, opt = c.layout(), c.options()
    n = c.q.shape[0]
    all_ = torch.full((n, 9, 32), 5.0, dtype=dtype, device="cuda")
    q, k, v = all_[:, :4], all_[:, 4:6], all_[:, 6:8]
    q.copy_(c.q), k.copy_(c.k), v.copy_(c.v)
    kept, want = fs.fs_jagged_attention(ctx, q, k, v, **lay, **opt, keep=True), c.forward(ctx, keep=True)
    for name in want:
        assert torch.equal(kept[name], want[name]), name
    grads = torch.full((n, 9, 32), -7.0, dtype=dtype, device="cuda")
    out = {"dq": grads[:, :4], "dk": grads[:, 4:6], "dv": grads[:, 6:8]}
    got = fs.fs_jagged_attention_backward(ctx, c.dout.cuda(), kept, q, k, v, **lay, **opt, out=out)
    ref = c.backward(ctx, want)
    for name in ref:
        assert torch.equal(got[name], ref[name]), name
    assert bool((grads[:, 8] == -7.0).all()) and torch.equal(grads[:, 4:6], ref["dk"])


@pytest.mark.parametrize("causal", [True, False])
def test_gradients_against_differences(ctx, causal):
    c = Case([40, 1, 75], heads=2, kv_heads=1, width=16, causal=causal)
    kept = c.forward(ctx, keep=True)
    got = c.backward(ctx, kept)
    scale = c.q.shape[2] ** -0.5
    leaves = {"q": c.q.double(), "k": c.k.double(), "v": c.v.double(), "bias": c.bias.double()}

    def loss(t):
        o = attention(t["q"], t["k"], t["v"], c.lens_q, c.lens_k, c.rooms, t["bias"], c.bucket_of, c.causal, scale, F32)["out"][0]
        return float((o * c.dout.double()).sum())

    for name, leaf in leaves.items():
        way = torch.randn(leaf.shape, generator=torch.Generator().manual_seed(3), dtype=torch.float64)
        ends = [loss({**leaves, name: leaf + s * 1e-5 * way}) for s in (1, -1)]
        terms = got["d" + name].cpu().double() * way
        assert abs((ends[0] - ends[1]) / 2e-5 - float(terms.sum())) <= 1e-5 * float(terms.abs().sum()) + 1e-6, name


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("causal", [True, False])
def test_a_bias_that_hides(ctx, dtype, causal):
    """Buckets of -infinity: their pairs are not seen, and a row that meets nothing else sees nothing."""
    c = Case([100, 65, 1, 30], dtype=dtype, causal=causal, buckets=6, distances=20)
    c.bias[2, :] = -np.inf
    c.bias[0, 1] = -np.inf
    c.check(ctx)
    c.bias[:] = -np.inf
    got = c.check(ctx)
    assert bool((got["out"] == 0).all())
    back = c.backward(ctx, got)
    assert all(bool((back[n] == 0).all()) for n in back)
    c = Case([3, 2], [300, 600], dtype=dtype, causal=causal, buckets=6, distances=500)
    c.bias[1:4, :] = -np.inf
    c.check(ctx, grads=False, max_q=3)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("causal", [True, False])
def test_masks_of_a_types_lowest_value(ctx, dtype, causal):
    lows = [-4e4, -65504.0, -1e9, torch.finfo(BF16).min, torch.finfo(F32).min]
    for few in (0, 3):
        lens = ([3, 2, 1], [300, 600, 70]) if few else ([100, 65, 1, 30], None)
        c, d = (Case(*lens, dtype=dtype, causal=causal, buckets=8, distances=20) for _ in range(2))
        for i, low in enumerate(lows):
            c.bias[1 + i], d.bias[1 + i] = low, -np.inf
        c.bias[0, 1], d.bias[0, 1] = lows[-1], -np.inf
        got, want = c.forward(ctx, keep=True, max_q=few), d.forward(ctx, keep=True, max_q=few)
        back, ref = c.backward(ctx, got), d.backward(ctx, want)
        for x, y in ((got, want), (back, ref)):
            assert all(torch.equal(x[n], y[n]) for n in y if y[n] is not None)
        if not few:
            d.check(ctx)
    # low, but not that low: what a row meets nothing else of is what it sees
    c = Case([100, 65, 1, 30], dtype=dtype, causal=causal, buckets=3, distances=20)
    c.bias[:] = -1e4
    c.check(ctx)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("shift", [-3000.0, -200.0, 200.0, 3000.0])
def test_scores_far_from_zero(ctx, dtype, shift):
    """All scores of a row far below or above zero, in the first tile and in later ones."""
    c = Case([100, 300], dtype=dtype, buckets=3, distances=200)
    c.bias += shift
    c.check(ctx)
    c.bias += torch.tensor([0.0, shift, -shift])[:, None]
    c.check(ctx)
    c = Case([2, 1], [300, 700], dtype=dtype, buckets=3, distances=200)
    c.bias += shift
    c.check(ctx, grads=False, max_q=2)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), float("-inf")])
@pytest.mark.parametrize("what", ["q", "k", "v", "dout"])
def test_what_is_not_seen_does_not_reach(ctx, dtype, bad, what):
    """A value that is no number in a row of one user: rows before it, and other users, are as they are without it."""
    def build():
        return Case([20, 150, 40], dtype=dtype, heads=2, kv_heads=2, width=32)

    clean, c = build(), build()
    at = 20 + 100                                            # row 100 of the second user
    getattr(c, what)[at, 1, 7] = bad
    one, two = clean.forward(ctx, keep=True), c.forward(ctx, keep=True)
    b1, b2 = clean.backward(ctx, one), c.backward(ctx, two)
    before = [r for r in range(210) if not 120 <= r < 170]
    for name in ("out", "lse"):
        x, y = (t[name] if name == "out" else t[name].t() for t in (one, two))
        assert torch.equal(x[before], y[before]), name
        assert torch.equal(x[:, 0], y[:, 0]), name          # the other head
    assert torch.equal(b1["dq"][before], b2["dq"][before])
    # keys are reached by the rows that see them: those behind row 100 are not reached by its q and dout, and the keys of
    # other users by nothing
    other = [r for r in range(210) if not 20 <= r < 170]
    for name in ("dk", "dv"):
        assert torch.equal(b1[name][other], b2[name][other]), name
        if what in ("q", "dout"):
            behind = list(range(121, 170))
            assert torch.equal(b1[name][behind], b2[name][behind]), name
    if what == "v":
        # the rows that see it have it in its column, and nothing in the others
        y, x = two["out"][120:170, 1], one["out"][120:170, 1]
        cols = [i for i in range(32) if i != 7]
        assert torch.equal(x[:, cols], y[:, cols])
        assert bool(y[:, 7].isnan().all() if np.isnan(bad) else (y[:, 7] == bad).all())
    if what == "dout":
        y, x = b2["dv"][20:121, 1], b1["dv"][20:121, 1]
        cols = [i for i in range(32) if i != 7]
        assert torch.equal(x[:, cols], y[:, cols])
        assert bool(y[:, 7].isnan().all() if np.isnan(bad) else (y[:, 7] == bad).all())
    if what == "k" and np.isnan(bad):
        assert bool(two["out"][120:170, 1].isnan().all())


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
def test_what_lies_beside_the_keys_in_use_does_not_reach(ctx, dtype, bad):
    """Unused rows of a cache, and keys ahead of the first of several new rows."""
    c = Case([2, 1, 3], [300, 40, 70], [320, 64, 70], dtype=dtype, heads=4, kv_heads=2, width=64)
    one = {m: c.forward(ctx, max_q=m)["out"] for m in (0, 3)}
    for t in (c.k, c.v):
        t[300:320], t[360:384] = bad, bad                # beyond the users' 300 and 40 keys
    for m in (0, 3):
        assert torch.equal(c.forward(ctx, max_q=m)["out"], one[m])
    c.v[384 + 69, :, 3] = bad                            # the last key of the third user, seen by its last row only
    for m in (0, 3):
        got = c.forward(ctx, max_q=m)["out"]
        assert torch.equal(got[:5], one[m][:5])
        assert not bool(got[5, :, 3].isfinite().any()) and torch.equal(got[5, :, 4:], one[m][5, :, 4:])


def test_rows_far_apart(ctx):
    """Addresses beyond 2^31 elements and beyond 2^32 bytes."""
    stride, n = 1 << 22, 700
    big = torch.empty(n * stride, dtype=BF16, device="cuda").view(n, stride)
    c = Case([100, 600], heads=2, kv_heads=2, width=32, dtype=BF16)
    parts = [big[:, 64 * i:64 * i + 64].unflatten(1, (2, 32)) for i in range(6)]
    for to, x in zip(parts, (c.q, c.k, c.v)):
        to.copy_(x)
    lay, opt = c.layout(), c.options()
    want = c.forward(ctx, keep=True)
    kept = fs.fs_jagged_attention(ctx, *parts[:3], **lay, **opt, keep=True)
    assert torch.equal(kept["out"], want["out"])
    out = dict(zip(("dq", "dk", "dv"), parts[3:]))
    got, ref = fs.fs_jagged_attention_backward(ctx, c.dout.cuda(), kept, *parts[:3], **lay, **opt, out=out), c.backward(ctx, want)
    for name in ref:
        assert torch.equal(got[name], ref[name]), name
    s = Case([1, 2], [100, 600], heads=2, kv_heads=2, width=32, dtype=BF16)
    parts[1].copy_(s.k), parts[2].copy_(s.v)
    got = fs.fs_jagged_attention(ctx, s.q.cuda(), parts[1], parts[2], **s.layout(), **s.options(), max_q=2)
    assert torch.equal(got["out"], s.forward(ctx, max_q=2)["out"])


def test_nothing_to_do(ctx):
    for lens_q, lens_k in (([], []), ([0, 0], [0, 0]), ([0, 0], [5, 9]), ([4, 1], [0, 0])):
        c = Case(lens_q, lens_k, heads=2, kv_heads=1)
        got = c.forward(ctx, keep=True)
        assert bool((got["out"] == 0).all())
        back = c.backward(ctx, got, out={"dbias": torch.full((8, 2), 3.0, device="cuda")})
        assert all(bool((t == 0).all()) for t in back.values())
        assert bool((c.forward(ctx, max_q=4)["out"] == 0).all())


def test_a_bucket_that_is_none(ctx):
    c = Case([80, 100], buckets=5, distances=60)
    c.bucket_of[30], c.bucket_of[50] = 5, -1
    d = Case([80, 100], buckets=6, distances=60)             # what it counts as: a bucket of its own, of zero
    d.bias[:5], d.bias[5] = c.bias, 0.0
    d.bucket_of[:] = c.bucket_of
    d.bucket_of[30] = d.bucket_of[50] = 5
    for t in ("q", "k", "v", "dout"):
        getattr(d, t).copy_(getattr(c, t))
    got, want = c.forward(ctx, keep=True), d.forward(ctx, keep=True)
    assert fs.fs_check_async(ctx) == fs.FS_ERANGE
    assert torch.equal(got["out"], want["out"])
    back, ref = c.backward(ctx, got), d.backward(ctx, want)
    assert fs.fs_check_async(ctx) == fs.FS_ERANGE
    assert torch.equal(back["dbias"], ref["dbias"][:5]) and torch.equal(back["dk"], ref["dk"])
    few = Case([2, 1], [80, 100], buckets=5, distances=60)
    few.bucket_of[30] = 1 << 20
    few.forward(ctx, max_q=2)
    assert fs.fs_check_async(ctx) == fs.FS_ERANGE


@pytest.mark.parametrize("offs", [[0, 50, 40, 100], [5, 50, 70, 100], [0, 50, 70, 90], [0, 50, 70, 120], [0, -10, 70, 100],
                                  [0, 1 << 50, 70, 100], [1 << 62, 50, 1 << 63 - 1, -(1 << 62)], [0, 110, 110, 100]])
@pytest.mark.parametrize("which", ["q", "kv", "both"])
def test_boundaries_that_do_not_fit_are_reported(ctx, offs, which):
    c = Case([50, 20, 30], heads=2, kv_heads=1, dtype=BF16)
    good, bad = offsets(c.lens_q).cuda(), torch.tensor(offs, dtype=torch.int64).cuda()
    lay = (bad if which != "kv" else good, bad if which != "q" else good)
    args = (c.q.cuda(), c.k.cuda(), c.v.cuda(), *lay)
    fs.fs_jagged_attention(ctx, *args, **c.options())
    assert fs.fs_check_async(ctx) == fs.FS_ERANGE and "offsets" in ctx.last_error()
    fs.fs_jagged_attention(ctx, *args, **c.options(), max_q=8)
    assert fs.fs_check_async(ctx) == fs.FS_ERANGE
    kept = c.forward(ctx, keep=True)
    assert fs.fs_check_async(ctx) == fs.FS_OK
    fs.fs_jagged_attention_backward(ctx, c.dout.cuda(), kept, *args, **c.options())
    assert fs.fs_check_async(ctx) == fs.FS_ERANGE


def test_lengths_that_do_not_fit_are_reported(ctx):
    for lens in ([-1, 5], [11, 5], [10, 1 << 40]):
        c = Case([2, 2], [10, 10], [10, 10])
        c.lens_k = lens
        c.forward(ctx, max_q=2)
        assert fs.fs_check_async(ctx) == fs.FS_ERANGE
        c.forward(ctx)
        assert fs.fs_check_async(ctx) == fs.FS_ERANGE


def test_more_rows_than_announced(ctx):
    c = Case([2, 5, 1], [40, 300, 600], dtype=BF16)
    want = c.forward(ctx)["out"]
    out = torch.full_like(want, 7.0)
    got = c.forward(ctx, max_q=2, out={"out": out})["out"]
    assert fs.fs_check_async(ctx) == fs.FS_ERANGE
    assert bool((got[2:7] == 7.0).all())                     # its rows are left as they were, the others are there
    for rows in (slice(0, 2), slice(7, 8)):
        assert torch.allclose(got[rows].float(), want[rows].float(), rtol=2 ** -6, atol=2 ** -6)


def test_the_same_again_and_on_other_streams(ctx):
    c = Case([700, 300, 5, 64], heads=4, kv_heads=2, width=64, dtype=BF16, distances=100)
    few = Case([1, 2], [3000, 700], heads=4, kv_heads=2, width=64, dtype=BF16)
    kept = c.forward(ctx, keep=True)
    want, first = c.backward(ctx, kept), few.forward(ctx, max_q=2)["out"]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    for _ in range(3):
        runs = []
        for s in streams:
            s.wait_stream(torch.cuda.current_stream())
            with torch.cuda.stream(s):
                k = c.forward(ctx, keep=True)
                runs.append((k, c.backward(ctx, k), few.forward(ctx, max_q=2)["out"]))
        torch.cuda.synchronize()
        for k, back, out in runs:
            assert torch.equal(k["out"], kept["out"]) and torch.equal(out, first)
            for name in want:
                assert torch.equal(back[name], want[name]), name
    # a stream that is named instead of being current
    lay = few.layout()
    args = (few.q.cuda(), few.k.cuda(), few.v.cuda(), lay["q_offsets"], lay["kv_offsets"])
    torch.cuda.synchronize()
    for s in (streams[0], streams[1].cuda_stream):
        got = fs.fs_jagged_attention(ctx, *args, **few.options(), max_q=2, stream=s)["out"]
        torch.cuda.synchronize()
        assert torch.equal(got, first)


def test_captured_and_replayed(ctx):
    """Two graphs of the same context and buffers, replayed in turn with eager calls between them."""
    c = Case([300, 5, 129], heads=4, kv_heads=2, width=32, dtype=BF16)
    few = Case([1, 2], [3000, 700], heads=4, kv_heads=2, width=32, dtype=BF16)
    lay, opt, flay, fopt = c.layout(), c.options(), few.layout(), few.options()
    q, k, v, dout = (t.cuda() for t in (c.q, c.k, c.v, c.dout))
    fq, fk, fv = (t.cuda() for t in (few.q, few.k, few.v))

    def train():
        kept = fs.fs_jagged_attention(ctx, q, k, v, **lay, **opt, keep=True)
        return {"out": kept["out"], **fs.fs_jagged_attention_backward(ctx, dout, kept, q, k, v, **lay, **opt)}

    def serve():
        return fs.fs_jagged_attention(ctx, fq, fk, fv, **flay, **fopt, max_q=2)

    train(), serve()
    torch.cuda.synchronize()
    graphs = []
    for call in (train, serve, train):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            res = call()
        graphs.append((graph, call, res))
    for turn in range(4):
        for t in (q, k, v, dout, fq, fk, fv):
            t.copy_(torch.randn(t.shape, generator=torch.Generator().manual_seed(turn)).to(t.dtype))
        for graph, _, _ in graphs:
            graph.replay()
        for graph, call, res in graphs:
            want = call()
            for name in want:
                assert torch.equal(res[name], want[name]), (turn, name)


def test_captured_with_large_tables_before_any_other_call(ctx):
    """Kernels that ask for more LDS than they have unasked, first of all in a capture; replayed on other inputs."""
    c = Case([150, 65], width=128, heads=2, kv_heads=1, buckets=512, distances=4000, causal=False)
    lay, opt = c.layout(), c.options()
    q, k, v, dout = (t.cuda() for t in (c.q, c.k, c.v, c.dout))

    def train():
        kept = fs.fs_jagged_attention(ctx, q, k, v, **lay, **opt, keep=True)
        return {"out": kept["out"], **fs.fs_jagged_attention_backward(ctx, dout, kept, q, k, v, **lay, **opt)}

    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        res = train()
    for turn in range(3):
        for t in (q, k, v, dout):
            t.copy_(torch.randn(t.shape, generator=torch.Generator().manual_seed(turn)).to(t.dtype))
        graph.replay()
        want = train()
        for name in want:
            assert torch.equal(res[name], want[name]), (turn, name)


@pytest.mark.parametrize("users", [64, 65, 66, 129, 200, 256, 1000, 4097])
def test_many_users(ctx, users):
    """Every user is found, the last ones among them, by tiles of rows, of keys and by row."""
    lens = [(7 * u) % 5 for u in range(users)]
    Case(lens, heads=1, kv_heads=1, width=8, dtype=BF16).check(ctx)
    c = Case([1] * users, [260 + u % 3 for u in range(users)], heads=1, kv_heads=1, width=8, dtype=BF16, buckets=0)
    got = c.forward(ctx, max_q=1, out={"out": torch.full_like(c.q, float("nan")).cuda()})["out"]
    assert_bounded(got, *c.want(False)["out"], "few")

"""Pairs that a bias hides, where what they would bring is no number: nothing of it reaches the row, the key or the bias."""
import numpy as np
import pytest
import torch

import paper_2604_24073_amd as fs
from test_gpu_jagged_attention import BF16, F32, Case

pytestmark = pytest.mark.gpu

BADS = [float("nan"), float("inf"), float("-inf")]


@pytest.fixture(scope="module")
def ctx():
    c = fs.Context(max_ids=1024)
    yield c
    assert fs.fs_check_async(c) == fs.FS_OK, c.last_error()
    c.close()


def build(lens_q, lens_k, width, dtype, causal):
    """Two heads; head 1 sees the distances of buckets 0 and 2, and not those of 1 and of 3, the table's last on either side."""
    c = Case(lens_q, lens_k, dtype=dtype, causal=causal, heads=2, kv_heads=2, width=width, buckets=4, distances=90, seed=3)
    d = torch.arange(90)
    near = torch.where(d < 7, 0, torch.where(d < 33, 1, torch.where(d < 80, 2, 3))).to(torch.int32)
    c.bucket_of = near if causal else torch.cat([near.flip(0)[:-1], near])
    c.bias[1, 1] = c.bias[3, 1] = -np.inf
    return c


def sees(c, user):
    """[rows, keys] of a user, head 1."""
    nq, nk = c.lens_q[user], c.lens_k[user]
    d = torch.arange(nq)[:, None] + (nk - nq) - torch.arange(nk)[None, :]
    size = len(c.bucket_of)
    bucket = c.bucket_of[d.clamp(0, size - 1) if c.causal else d.clamp(-(size // 2), size // 2) + size // 2].long()
    seen = c.bias[:, 1][bucket] > -np.inf
    return seen & (d >= 0) if c.causal else seen


@pytest.mark.parametrize("dtype,lens,width", [(F32, [30, 300], 32), (BF16, [30, 300], 32), (BF16, [30, 1300], 64), (F32, [5, 210], 128)])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("bad", BADS)
@pytest.mark.parametrize("what", ["q", "k", "v", "dout"])
def test_a_row_or_key_behind_a_hidden_bucket(ctx, dtype, lens, width, causal, bad, what):
    clean, c = (build(lens, None, width, dtype, causal) for _ in range(2))
    at = lens[1] // 2
    getattr(c, what)[lens[0] + at, 1, 5] = bad
    one, two = clean.forward(ctx, keep=True), c.forward(ctx, keep=True)
    b1, b2 = clean.backward(ctx, one), c.backward(ctx, two)
    pairs = sees(c, 1)
    rows = torch.zeros(lens[1], dtype=torch.bool)
    if what in ("k", "v"):
        rows |= pairs[:, at]                                 # the rows that have the key among theirs
    else:
        rows[at] = True
    keys = pairs[rows].any(0)                                # the keys that such a row sees
    if what in ("k", "v"):
        keys[at] = True
    mine = slice(lens[0], lens[0] + lens[1])
    free_rows, free_keys = (~rows).nonzero()[:, 0], (~keys).nonzero()[:, 0]
    assert len(free_rows) > 30 and (len(free_keys) > 30 or what in ("k", "v"))
    for name, x, y in (("out", one["out"], two["out"]), ("lse", one["lse"].t()[..., None], two["lse"].t()[..., None]),
                       ("dq", b1["dq"], b2["dq"]), ("dk", b1["dk"], b2["dk"]), ("dv", b1["dv"], b2["dv"])):
        assert torch.equal(x[:, 0], y[:, 0]) and torch.equal(x[:lens[0]], y[:lens[0]]), name
        free = (free_rows if name in ("out", "lse", "dq") else free_keys).cuda()
        assert torch.equal(x[mine, 1][free], y[mine, 1][free]), name
    for x in (b1["dbias"], b2["dbias"]):
        assert bool((x[[1, 3], 1] == 0).all())
    assert torch.equal(b1["dbias"][:, 0], b2["dbias"][:, 0])


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("bad", BADS)
def test_a_head_that_sees_nothing(ctx, dtype, causal, bad):
    """Every value of the head's rows is no number, and every bias of it hides."""
    c = build([70, 1, 200], None, 32, dtype, causal)
    c.bias[:, 1] = -1e9
    want = c.forward(ctx, keep=True)
    ref = c.backward(ctx, want)
    for t in (c.q, c.k, c.v, c.dout):
        t[:, 1] = bad
    got = c.forward(ctx, keep=True)
    back = c.backward(ctx, got)
    assert bool((got["out"][:, 1] == 0).all()) and bool((got["lse"][1] == -np.inf).all())
    for x, y in ((want, got), (ref, back)):
        for name in x:
            assert torch.equal(x[name], y[name]), name
    assert all(bool((back[n][:, 1] == 0).all()) for n in back)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("bad", BADS)
@pytest.mark.parametrize("what", ["q", "k", "v"])
def test_few_rows(ctx, dtype, causal, bad, what):
    """Caches of one chunk and of several, in the form for few rows and in the other."""
    for keys in ([85, 110], [600, 1400]):
        clean, c = (build([3, 2], keys, 64, dtype, causal) for _ in range(2))
        at = keys[1] - 20                                    # 18 and 19 distances from the second user's rows
        seen = sees(c, 1)
        assert not bool(seen[:, at].any())
        if what == "q":
            c.bias[:, 1] = clean.bias[:, 1] = -np.inf
            c.q[:, 1] = bad
        else:
            getattr(c, what)[keys[0] + at, 1, 9] = bad
            getattr(c, what)[:10, 1, 9] = bad                # the far side of the first user's cache
            if keys[0] == 85:
                getattr(c, what)[:10, 1, 9] = 1.0            # near enough to be seen
                getattr(clean, what)[:10, 1, 9] = 1.0
        for max_q in (3, 0):
            one, two = clean.forward(ctx, keep=True, max_q=max_q), c.forward(ctx, keep=True, max_q=max_q)
            for name in one:
                assert torch.equal(one[name], two[name]), (keys, max_q, name)
        if what == "q":
            assert bool((two["out"][:, 1] == 0).all())

"""What bf16 rows lose and what they do not: the unrounded out and the bias's gradient are held in 32 bits all the way, from P in
more than one term of bf16 and from an out that has not been rounded.  Bounds by element add up magnitudes and are too wide to
tell; these are on the error relative to a result's norm, and a plain form with the roundings put in shows that they tell."""
import pytest
import torch

import paper_2604_24073_amd as fs
from encoder_refs import attention
from test_gpu_jagged_attention import BF16, F32, Case

# Roundings in 32 bits add up like the root of their number.  A score is a sum of up to 129 terms about a size of up to 20 (the
# rows' scores and what they are less by), cut off instead of rounded: sqrt(129) 2^-23 20 = 2.7e-5 in the power, that much of P,
# in out as in P.  P as one term of bf16 is off by 2^-9 / sqrt(3) = 1.1e-3 of itself.
OUT = 1e-4
# The errors of a row's powers that are common to its keys leave its dS in sum; what is left are those of D and dO V^T, sums of up
# to 128 terms: sqrt(128) 2^-23 = 1.3e-6 of themselves, and as many independent ones in the sum of a bucket as values.  A few of
# them: 1e-5.  An out made of P in one term, or a rounded one, is off by about 1e-3 of itself, and D with it.
DBIAS = 1e-5


def case(dtype, width, causal, lens=(1100, 700, 60), seed=5):
    c = Case(lens, heads=2, kv_heads=1, width=width, dtype=dtype, causal=causal, buckets=6, distances=300, seed=seed)
    d = torch.arange(300)
    near = (d.float() + 1).log2().mul(0.8).clamp(max=5).to(torch.int32)
    c.bucket_of = near if causal else torch.cat([near.flip(0)[:-1], near])
    return c


def off(got, want):
    return float((got.detach().cpu().double() - want).norm() / want.norm())


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("width", [32, 64, 128])
def test_out_and_the_gradient_of_the_bias(dtype, causal, width):
    ctx = fs.Context(max_ids=1024)
    for lens in ((1100, 700, 60), (300, 250, 200, 1)):
        c = case(dtype, width, causal, lens)
        want = c.want()
        kept = c.forward(ctx, keep=True)
        unrounded = kept["out_f32"] if dtype == BF16 else kept["out"]
        assert off(unrounded, want["out"][0]) <= OUT
        assert off(kept["lse"], want["lse"][0]) <= OUT
        dbias, ref = c.backward(ctx, kept)["dbias"], want["dbias"][0]
        for head in range(2):
            assert off(dbias[:, head], ref[:, head]) <= DBIAS, (lens, head)
    assert fs.fs_check_async(ctx) == fs.FS_OK
    ctx.close()


def plain(c, terms=0, out_dtype=None, lost=0):
    """(out, dbias) in 64 bits with roundings put in: P in so many terms of bf16 where it makes out (0: as it is), the out that D
    is made of, and pairs left out of the bias's gradient."""
    scale = c.q.shape[2] ** -0.5
    outs, dbias, at = [], torch.zeros(c.bias.shape, dtype=torch.float64), 0
    for n in c.lens_q:
        rows = slice(at, at + n)
        d = torch.arange(n)[:, None] - torch.arange(n)[None, :]
        size = len(c.bucket_of)
        bucket = c.bucket_of[d.clamp(0, size - 1) if c.causal else d.clamp(-(size // 2), size // 2) + size // 2].long()
        heads = []
        for h in range(2):
            q, k, v, do = (t.double() for t in (c.q[rows, h], c.k[rows, 0], c.v[rows, 0], c.dout[rows, h]))
            s = scale * (q @ k.T) + c.bias.double()[:, h][bucket]
            p = torch.softmax(s.masked_fill(d < 0, float("-inf")) if c.causal else s, 1)
            left, used = p, p if not terms else torch.zeros_like(p)
            for _ in range(terms):
                term = left.to(BF16).double()
                left, used = left - term, used + term
            o = used @ v
            heads.append(o)
            D = (do * (o if out_dtype is None else o.to(out_dtype).double())).sum(1, keepdim=True)
            ds = p * (do @ v.T - D)
            if lost:
                ds[::lost, :1] = 0
            dbias[:, h].index_add_(0, bucket.reshape(-1), ds.reshape(-1))
        outs.append(torch.stack(heads, 1))
        at += n
    return torch.cat(outs), dbias


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("width", [32, 64])
def test_the_bounds_tell(causal, width):
    c = case(BF16, width, causal)
    want = attention(c.q.double(), c.k.double(), c.v.double(), c.lens_q, c.lens_k, c.rooms, c.bias.double(), c.bucket_of, causal,
                     width ** -0.5, BF16, c.dout.double())
    out, dbias = want["out"][0], want["dbias"][0]
    for terms in (0, 3):
        o, b = plain(c, terms)
        assert off(o, out) <= OUT / 10 and all(off(b[:, h], dbias[:, h]) <= DBIAS / 10 for h in range(2))
    o, b = plain(c, terms=1)
    assert off(o, out) > 5 * OUT and all(off(b[:, h], dbias[:, h]) > 5 * DBIAS for h in range(2))
    _, b = plain(c, out_dtype=BF16)
    assert all(off(b[:, h], dbias[:, h]) > 5 * DBIAS for h in range(2))
    _, b = plain(c, lost=100)
    assert all(off(b[:, h], dbias[:, h]) > 5 * DBIAS for h in range(2))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("width", [32, 64, 128])
def test_few_rows_against_caches(dtype, causal, width):
    """The form for few rows keeps P's bits too, and so does a backward pass behind it."""
    ctx = fs.Context(max_ids=1024)
    lens_q, lens_k = [4] * 8, [60, 300, 700, 1500, 90, 257, 256, 33]
    c = Case(lens_q, lens_k, [n + 5 for n in lens_k], heads=2, kv_heads=1, width=width, dtype=dtype, causal=causal, buckets=6,
             distances=300, seed=9)
    c.bucket_of = case(dtype, width, causal).bucket_of
    want = c.want()
    kept = c.forward(ctx, keep=True, max_q=4)
    unrounded = kept["out_f32"] if dtype == BF16 else kept["out"]
    assert off(unrounded, want["out"][0]) <= OUT and off(kept["lse"], want["lse"][0]) <= OUT
    dbias, ref = c.backward(ctx, kept)["dbias"], want["dbias"][0]
    for head in range(2):
        assert off(dbias[:, head], ref[:, head]) <= DBIAS, head
    assert fs.fs_check_async(ctx) == fs.FS_OK
    ctx.close()

"""Few rows of very many users against their caches: more rows and heads than a launch has threads for."""
import pytest
import torch

import paper_2604_24073_amd as fs
from encoder_refs import assert_bounded, attention

pytestmark = pytest.mark.gpu


def test_more_rows_and_heads_than_a_launch_has_wavefronts():
    """2^24 rows of 4 heads, each a wavefront's where caches are put together.  The first user and the last have caches of
    several chunks, every other one a single key, whose value is what its rows get."""
    users, rows, heads, width, long = 1 << 20, 16, 4, 8, 5000
    ctx = fs.Context(max_ids=1024)
    gen = torch.Generator(device="cuda").manual_seed(1)
    n_q, n_kv = users * rows, users - 2 + 2 * long
    assert n_q * heads >= 1 << 26
    q = torch.randn(n_q, heads, width, generator=gen, device="cuda", dtype=torch.bfloat16)
    k, v = (torch.randn(n_kv, heads, width, generator=gen, device="cuda", dtype=torch.bfloat16) for _ in range(2))
    q_offsets = torch.arange(users + 1, device="cuda") * rows
    kv_offsets = torch.arange(users + 1, device="cuda") + (long - 1)
    kv_offsets[0], kv_offsets[-1] = 0, n_kv
    out = torch.full_like(q, 9.0)
    got = fs.fs_jagged_attention(ctx, q, k, v, q_offsets, kv_offsets, causal=False, max_q=rows, out={"out": out})["out"]
    by_user = got.view(users, rows, heads, width)
    assert torch.equal(by_user[1:-1], v[long:n_kv - long, None].expand(-1, rows, -1, -1))
    for user, keys in ((0, slice(0, long)), (users - 1, slice(n_kv - long, n_kv))):
        rows_of = slice(user * rows, (user + 1) * rows)
        want = attention(q[rows_of].cpu().double(), k[keys].cpu().double(), v[keys].cpu().double(), [rows], [long], [long], None,
                         None, False, width ** -0.5, torch.bfloat16)["out"]
        assert_bounded(got[rows_of], *want, f"user {user}")
    assert fs.fs_check_async(ctx) == fs.FS_OK
    ctx.close()

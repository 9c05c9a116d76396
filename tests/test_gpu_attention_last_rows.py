"""The rows of a workgroup behind a user's last one are none: a key that is no number reaches the biases of the distances from rows
that see it, and of no others."""
import pytest
import torch

import paper_2604_24073_amd as fs
from test_gpu_jagged_attention import BF16, F32, Case

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    c = fs.Context(max_ids=1024)
    yield c
    assert fs.fs_check_async(c) == fs.FS_OK, c.last_error()
    c.close()


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("width", [32, 64, 128])
@pytest.mark.parametrize("rows,keys", [(5, 5), (70, 70), (3, 40), (130, 130), (600, 600)])
@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
def test_biases_that_no_pair_meets(ctx, dtype, causal, width, rows, keys, bad):
    distances, group = 1000, 1 if rows < 600 else 2                # a bucket has one distance, or two neighbouring ones
    c = Case([rows], [keys], heads=2, kv_heads=1, width=width, dtype=dtype, causal=causal, buckets=1024, distances=distances)
    d = torch.arange(distances) if causal else torch.arange(-distances + 1, distances)
    c.bucket_of = ((d // group) % 1024).to(torch.int32)            # distances that are 1024 buckets apart: 0 and the far side's
    met = torch.arange(rows)[:, None] + (keys - rows) - torch.arange(keys)[None, :]
    met = met[met >= 0] if causal else met.reshape(-1)
    meets = torch.zeros(1024, dtype=torch.bool)
    meets[(met // group) % 1024] = True
    for at in (3, keys - 1):
        c.k.copy_(torch.randn(c.k.shape, generator=torch.Generator().manual_seed(7)).to(dtype))
        c.k[at, 0, 5] = bad
        dbias = c.backward(ctx, c.forward(ctx, keep=True))["dbias"].cpu()
        assert bool((dbias[~meets] == 0).all()) and int((~meets).sum()) > 100, at

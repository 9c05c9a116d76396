"""Two threads of the host with a context each, whose tables differ and whose kernels ask for different amounts of LDS."""
import threading

import pytest
import torch

import paper_2604_24073_amd as fs
from test_gpu_jagged_attention import F32, Case

pytestmark = pytest.mark.gpu


def test_tables_of_different_sizes_at_once():
    cases = [Case([70, 33], width=128, heads=2, kv_heads=1, buckets=b, distances=d, causal=False, dtype=F32, seed=b)
             for b, d in ((1024, 4096), (64, 700))]
    contexts = [fs.Context(max_ids=1024) for _ in cases]
    inputs = [([t.cuda() for t in (c.q, c.k, c.v)], c.dout.cuda(), c.layout(), c.options()) for c in cases]

    def step(i):
        qkv, dout, layout, options = inputs[i]
        kept = fs.fs_jagged_attention(contexts[i], *qkv, **layout, **options, keep=True)
        return {"out": kept["out"], **fs.fs_jagged_attention_backward(contexts[i], dout, kept, *qkv, **layout, **options)}

    want = [step(i) for i in range(2)]
    torch.cuda.synchronize()
    got, errors = [[], []], []

    def loop(i):
        try:
            with torch.cuda.stream(torch.cuda.Stream()):
                for _ in range(100):
                    got[i].append(step(i))
        except Exception as e:                                   # noqa: BLE001 - reported by the thread that started this one
            errors.append(e)

    threads = [threading.Thread(target=loop, args=(i,)) for i in range(2)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    torch.cuda.synchronize()
    assert not errors
    for i in range(2):
        assert len(got[i]) == 100
        for res in got[i]:
            for name, t in want[i].items():
                assert torch.equal(res[name], t), (i, name)
    for c in contexts:
        assert fs.fs_check_async(c) == fs.FS_OK
        c.close()

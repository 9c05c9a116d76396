"""Calls of the history encoder on a stream that is named, beside calls on the current stream that have not ended: each has
inputs of its own, and results that are its own."""
import pytest
import torch

import paper_2604_24073_amd as fs

pytestmark = pytest.mark.gpu

F32, BF16, EPS = torch.float32, torch.bfloat16, 1e-6


@pytest.fixture(scope="module")
def ctx():
    c = fs.Context(max_ids=1024)
    yield c
    assert fs.fs_check_async(c) == fs.FS_OK, c.last_error()
    c.close()


def rnd(shape, dtype, seed):
    return torch.randn(shape, generator=torch.Generator().manual_seed(seed)).to(dtype).cuda()


def block_backward(ctx, seed):
    """A call of the backward pass, its stream left open."""
    n, dim = 40_000, 128
    a, g, dh = (rnd((n, dim), BF16, 10 * seed + i) for i in range(3))
    y, dy = (rnd((n, dim), F32, 10 * seed + i) for i in (3, 4))
    w = [rnd((dim,), F32, 10 * seed + i) for i in (5, 6, 7)]
    return lambda stream: fs.fs_block_norm_backward(ctx, dy, dh, a, g, y, *w, eps=EPS, stream=stream)


def attention(ctx, seed, way):
    rows, keys = ([1200] * 6, [1200] * 6) if way != "few rows" else ([2] * 6, [9000] * 6)
    q, dout = (rnd((sum(rows), 4, 64), BF16, 10 * seed + i) for i in (0, 1))
    k, v = (rnd((sum(keys), 2, 64), BF16, 10 * seed + i) for i in (2, 3))
    qo, ko = (torch.tensor([0] + [sum(x[:i + 1]) for i in range(6)], dtype=torch.int64).cuda() for x in (rows, keys))
    position = {"bias": rnd((16, 4), F32, 10 * seed + 4), "bucket_of": (torch.arange(400) // 25).to(torch.int32).cuda()}
    forward = lambda stream: fs.fs_jagged_attention(ctx, q, k, v, qo, ko, **position, keep=True,  # noqa: E731
                                                    max_q=2 if way == "few rows" else 0, stream=stream)
    if way != "backward":
        return forward
    kept = forward(None)
    return lambda stream: fs.fs_jagged_attention_backward(ctx, dout, kept, q, k, v, qo, ko, **position, stream=stream)


def calls_of(ctx, what, seed):
    return block_backward(ctx, seed) if what == "block" else attention(ctx, seed, what)


@pytest.mark.parametrize("handle", [False, True])
@pytest.mark.parametrize("what", ["block", "backward", "few rows", "forward"])
def test_beside_the_current_stream(ctx, what, handle):
    calls = [calls_of(ctx, what, seed) for seed in (1, 2)]
    want = [{k: t.clone() for k, t in call(None).items()} for call in calls]
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    named = side.cuda_stream if handle else side
    ahead = torch.randn(4096, 4096, device="cuda")
    for turn in range(4):
        for _ in range(3):
            ahead @ ahead                                        # what the current stream has ahead of its call
        got = [(0, calls[0](None)), (1, calls[1](named)), (0, calls[0](None)), (1, calls[1](named))]
        if turn % 2:
            got.append((1, calls[1](None)))
        torch.cuda.synchronize()
        for which, res in got:
            for name, t in want[which].items():
                assert torch.equal(res[name], t), (turn, which, name)
        del got, res, t


@pytest.mark.parametrize("what", ["block", "backward", "few rows"])
def test_scratch_is_of_the_named_streams_pool(ctx, what):
    """What a call leaves behind in torch's memory is behind on its own stream's side."""
    call = calls_of(ctx, what, 3)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())

    def segments(stream):
        return sum(s["total_size"] for s in torch.cuda.memory_snapshot() if s["stream"] == stream)

    torch.cuda.synchronize()
    torch.cuda.empty_cache()                                     # torch's streams may have been others' before
    before = [segments(s) for s in (side.cuda_stream, torch.cuda.current_stream().cuda_stream)]
    res = call(side)
    torch.cuda.synchronize()
    after = [segments(s) for s in (side.cuda_stream, torch.cuda.current_stream().cuda_stream)]
    assert after[0] > before[0] and after[1] == before[1]
    del res


def test_in_a_capture_that_forks(ctx):
    """The named stream joins a capture, and the graph holds both sides' work."""
    calls = [calls_of(ctx, "backward", seed) for seed in (4, 5)]
    want = [call(None) for call in calls]
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        main = torch.cuda.current_stream()
        side.wait_stream(main)
        got = [calls[0](None), calls[1](side)]
        main.wait_stream(side)
    for _ in range(3):
        for res in got:
            for t in res.values():
                t.fill_(3.0)
        graph.replay()
        torch.cuda.synchronize()
        for res, ref in zip(got, want):
            for name, t in ref.items():
                assert torch.equal(res[name], t), name
        calls[1](None)


@pytest.mark.parametrize("named", ["handle", "stream"])
def test_the_default_stream_named_beside_another(ctx, named):
    """Stream 0 by its handle and by torch's object, while another stream is the current one, which stays that."""
    calls = [calls_of(ctx, "backward", seed) for seed in (6, 7)]
    want = [{k: t.clone() for k, t in call(None).items()} for call in calls]
    torch.cuda.synchronize()
    side, default = torch.cuda.Stream(), torch.cuda.default_stream()
    with torch.cuda.stream(side):
        got = [calls[0](0 if named == "handle" else default), calls[1](None)]
        assert torch.cuda.current_stream() == side
    torch.cuda.synchronize()
    for res, ref in zip(got, want):
        for name, t in ref.items():
            assert torch.equal(res[name], t), name

"""The norms around a block and rows in 8 bits against their definitions in 64 bits, bound by bound."""
import numpy as np
import pytest
import torch

import paper_2604_24073_amd as fs
from encoder_refs import assert_within, block_norm, block_norm_backward, rows8

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16
EPS = 1e-5
# Roundings in 32 bits on the way to a value, each relative to its magnitude: a mean of squares sums 16 columns in a lane and
# at most 64 lanes in 6 steps (22, halved by the root), its root, reciprocal and product 3, the gate 6, products and the mean
# behind them (22 + 6).  Sums over rows take as many more as a lane adds up.
FORWARD, BACKWARD = 64, 128


@pytest.fixture(scope="module")
def ctx():
    c = fs.Context(max_ids=1024)
    yield c
    assert fs.fs_check_async(c) == fs.FS_OK
    c.close()


def rnd(shape, dtype=F32, seed=0, size=1.0):
    return (torch.randn(shape, generator=torch.Generator().manual_seed(seed)) * size).to(dtype)


def inputs(n, dim, rows_dt, dt, seed=1):
    t = {"x": rnd((n, dim), rows_dt, seed), "a": rnd((n, dim), dt, seed + 1, 0.7), "g": rnd((n, dim), dt, seed + 2, 2.0),
         "dy": rnd((n, dim), rows_dt, seed + 3), "dh": rnd((n, dim), dt, seed + 4)}
    for k, name in enumerate(("w_post", "scale", "w_pre")):
        t[name] = 1 + 0.3 * rnd((dim,), F32, seed + 5 + k)
    return t


def cuda(t):
    return {k: v.cuda() for k, v in t.items()}


def dbl(t):
    return {k: v.double() for k, v in t.items()}


SHAPES = [(1, 4, F32, F32), (1, 8, F32, BF16), (3, 20, F32, F32), (5, 8, BF16, BF16), (9, 36, F32, F32), (64, 32, BF16, F32),
          (127, 64, F32, BF16), (65, 100, F32, F32), (1000, 128, F32, BF16), (33, 200, BF16, BF16), (31, 256, F32, F32),
          (19, 264, F32, BF16), (7, 512, BF16, BF16), (257, 520, F32, BF16), (5, 1000, BF16, BF16), (11, 1024, F32, F32),
          (40_003, 32, F32, BF16), (70_001, 8, F32, F32)]


@pytest.mark.parametrize("n,dim,rows_dt,dt", SHAPES)
def test_forward(ctx, n, dim, rows_dt, dt):
    t = inputs(n, dim, rows_dt, dt)
    d, r = cuda(t), dbl(t)
    got = fs.fs_block_norm(ctx, d["x"], d["a"], d["g"], d["w_post"], d["scale"], d["w_pre"], eps=EPS)
    want = block_norm(r["x"], r["a"], r["g"], r["w_post"], r["scale"], r["w_pre"], EPS)
    assert got["y"].dtype == rows_dt and got["h"].dtype == dt and set(got) == {"y", "h"}
    for k in got:
        assert_within(got[k], *want[k], FORWARD, k)
    # the norm in front of the first block; no norm behind the last
    first = fs.fs_block_norm(ctx, d["x"], w_pre=d["w_pre"], eps=EPS, dtype=dt)
    assert set(first) == {"h"}
    assert_within(first["h"], *block_norm(r["x"], None, None, None, None, r["w_pre"], EPS)["h"], FORWARD, "first")
    last = fs.fs_block_norm(ctx, d["x"], d["a"], d["g"], d["w_post"], d["scale"], eps=EPS)
    assert set(last) == {"y"} and torch.equal(last["y"], got["y"])


@pytest.mark.parametrize("n,dim,rows_dt,dt", SHAPES)
def test_backward(ctx, n, dim, rows_dt, dt):
    t = inputs(n, dim, rows_dt, dt)
    t["y"] = rnd((n, dim), rows_dt, 77)
    d, r = cuda(t), dbl(t)
    w = (d["w_post"], d["scale"], d["w_pre"])
    more = n / 1024                                   # rows that a lane adds up
    for dy, dh, join in ((1, 1, 1), (0, 1, 1), (1, 0, 1), (1, 1, 0)):
        pick = lambda s, dy=dy, dh=dh, join=join: (s["dy"] if dy else None, s["dh"] if dh else None,  # noqa: E731
                                                   s["a"] if join else None, s["g"] if join else None, s["y"])
        got = fs.fs_block_norm_backward(ctx, *pick(d), *w, eps=EPS, rows_dtype=rows_dt)
        want = block_norm_backward(*pick(r), r["w_post"], r["scale"], r["w_pre"], EPS)
        assert set(got) == set(want)
        for k in got:
            assert_within(got[k], *want[k], BACKWARD + (more if k.startswith("dw") or k == "dscale" else 0), (dy, dh, join, k))


def test_gradients_against_differences(ctx):
    """The gradients as the slope of the 64-bit forward form along a direction: nothing of the formulas above in it."""
    n, dim = 13, 64
    t = inputs(n, dim, F32, F32, 40)
    d, r = cuda(t), dbl(t)
    y = fs.fs_block_norm(ctx, d["x"], d["a"], d["g"], d["w_post"], d["scale"], d["w_pre"], eps=EPS)["y"]
    got = fs.fs_block_norm_backward(ctx, d["dy"], d["dh"], d["a"], d["g"], y, d["w_post"], d["scale"], d["w_pre"], eps=EPS)

    def loss(v):
        f = block_norm(v["x"], v["a"], v["g"], v["w_post"], v["scale"], v["w_pre"], EPS)
        return float((f["y"][0] * r["dy"]).sum() + (f["h"][0] * r["dh"]).sum())

    for leaf, grad in (("x", "dx"), ("a", "da"), ("g", "dg"), ("w_post", "dw_post"), ("scale", "dscale"), ("w_pre", "dw_pre")):
        way = rnd(r[leaf].shape, seed=99).double()
        step = 1e-5
        ends = [loss({**r, leaf: r[leaf] + s * step * way}) for s in (1, -1)]
        slope = (ends[0] - ends[1]) / (2 * step)
        terms = got[grad].cpu().double() * way
        # third derivatives times step^2, cancellation in the difference, and the gradient's own roundings
        assert abs(slope - float(terms.sum())) <= 1e-5 * float(terms.abs().sum()) + 1e-6, leaf


def test_parts_of_one_tensor(ctx):
    """a and g, and their gradients, as column ranges of wider tensors; what lies beside them is left alone."""
    n, dim = 77, 64
    t = cuda(inputs(n, dim, F32, BF16))
    wide = torch.full((n, 200), 7.0, dtype=BF16, device="cuda")
    wide[:, 8:72], wide[:, 104:168] = t["a"], t["g"]
    w = (t["w_post"], t["scale"], t["w_pre"])
    want = fs.fs_block_norm(ctx, t["x"], t["a"], t["g"], *w, eps=EPS)
    got = fs.fs_block_norm(ctx, t["x"], wide[:, 8:72], wide[:, 104:168], *w, eps=EPS)
    assert torch.equal(got["y"], want["y"]) and torch.equal(got["h"], want["h"])
    back = fs.fs_block_norm_backward(ctx, t["dy"], t["dh"], t["a"], t["g"], want["y"], *w, eps=EPS)
    dwide = torch.full((n, 200), -3.0, dtype=BF16, device="cuda")
    out = {"da": dwide[:, 8:72], "dg": dwide[:, 104:168]}
    got = fs.fs_block_norm_backward(ctx, t["dy"], t["dh"], wide[:, 8:72], wide[:, 104:168], want["y"], *w, eps=EPS, out=out)
    for k in back:
        assert torch.equal(got[k], back[k]), k
    assert torch.equal(dwide[:, 8:72], back["da"]) and torch.equal(dwide[:, 104:168], back["dg"])
    for cols in (slice(0, 8), slice(72, 104), slice(168, 200)):
        assert bool((dwide[:, cols] == -3.0).all())


def test_in_place(ctx):
    t = cuda(inputs(300, 128, F32, BF16))
    w = (t["w_post"], t["scale"], t["w_pre"])
    want = fs.fs_block_norm(ctx, t["x"], t["a"], t["g"], *w, eps=EPS)
    back = fs.fs_block_norm_backward(ctx, t["dy"], t["dh"], t["a"], t["g"], want["y"], *w, eps=EPS)
    x, dy = t["x"].clone(), t["dy"].clone()
    got = fs.fs_block_norm(ctx, x, t["a"], t["g"], *w, eps=EPS, out={"y": x})
    assert torch.equal(x, want["y"]) and torch.equal(got["h"], want["h"])
    fs.fs_block_norm_backward(ctx, dy, t["dh"], t["a"], t["g"], x, *w, eps=EPS, out={"dx": dy})
    assert torch.equal(dy, back["dx"])


@pytest.mark.parametrize("dim", [8, 64, 1024])
def test_no_rows(ctx, dim):
    t = cuda(inputs(0, dim, F32, BF16))
    w = (t["w_post"], t["scale"], t["w_pre"])
    got = fs.fs_block_norm(ctx, t["x"], t["a"], t["g"], *w, eps=EPS)
    assert got["y"].shape == (0, dim)
    out = {k: torch.full((dim,), 9.0, device="cuda") for k in ("dw_post", "dscale", "dw_pre")}
    fs.fs_block_norm_backward(ctx, t["dy"], t["dh"], t["a"], t["g"], got["y"], *w, eps=EPS, out=out)
    assert all(bool((v == 0).all()) for v in out.values())


def test_values_that_are_no_numbers_stay_in_their_rows(ctx):
    n, dim = 66, 64
    t = inputs(n, dim, F32, F32)
    t["a"][3, 5], t["g"][10, 60], t["x"][33, 0], t["dh"][40, 1], t["dy"][50, 2] = (float("nan"), float("inf"), float("-inf"),
                                                                                  float("nan"), float("inf"))
    clean = cuda(inputs(n, dim, F32, F32))
    d = cuda(t)
    w = (d["w_post"], d["scale"], d["w_pre"])
    got = fs.fs_block_norm(ctx, d["x"], d["a"], d["g"], *w, eps=EPS)
    ref = fs.fs_block_norm(ctx, clean["x"], clean["a"], clean["g"], *w, eps=EPS)
    rest = [k for k in range(n) if k not in (3, 10, 33)]
    assert torch.equal(got["y"][rest], ref["y"][rest]) and torch.equal(got["h"][rest], ref["h"][rest])
    assert not got["h"][[3, 10, 33]].isfinite().all(1).any()
    back = fs.fs_block_norm_backward(ctx, d["dy"], d["dh"], d["a"], d["g"], got["y"], *w, eps=EPS)
    want = fs.fs_block_norm_backward(ctx, clean["dy"], clean["dh"], clean["a"], clean["g"], ref["y"], *w, eps=EPS)
    rest = [k for k in range(n) if k not in (3, 10, 33, 40, 50)]
    for k in ("dx", "da", "dg"):
        assert torch.equal(back[k][rest], want[k][rest]), k


def test_extremes(ctx):
    """Rows of zeros (their norm divides by the root of eps), tiny and huge rows, gates far out on both sides."""
    dim = 64
    t = inputs(6, dim, F32, F32)
    t["a"][0], t["x"][0] = 0.0, 0.0
    t["a"][1] *= 1e-30
    t["a"][2] *= 1e15
    t["g"][3], t["g"][4] = 200.0, -200.0
    d, r = cuda(t), dbl(t)
    got = fs.fs_block_norm(ctx, d["x"], d["a"], d["g"], d["w_post"], d["scale"], d["w_pre"], eps=EPS)
    want = block_norm(r["x"], r["a"], r["g"], r["w_post"], r["scale"], r["w_pre"], EPS)
    for k in got:
        assert_within(got[k], *want[k], FORWARD, k)
    back = fs.fs_block_norm_backward(ctx, d["dy"], d["dh"], d["a"], d["g"], got["y"], d["w_post"], d["scale"], d["w_pre"], eps=EPS)
    wantb = block_norm_backward(r["dy"], r["dh"], r["a"], r["g"], got["y"].cpu().double(), r["w_post"], r["scale"], r["w_pre"], EPS)
    for k in back:
        assert_within(back[k], *wantb[k], BACKWARD, k)


# ---- rows in 8 bits ------------------------------------------------------------------------------------------------------
def special_rows():
    x = rnd((40, 64), seed=9).numpy().copy()
    x[0] = 0.0
    x[1, :32] = 1e-45                              # below the smallest step
    x[2, 3] = 3.4e38
    x[3, :32], x[3, 0] = 0.25, 127.4999            # just below where the largest would round to 128 steps ...
    x[4, :32], x[4, 0] = 0.25, 127.5               # ... and there
    x[5, :32] = np.arange(32) + 0.5                # ties
    x[5, 31] = 64.0
    x[6, 7], x[7, 40], x[8, 33] = np.inf, np.nan, -np.inf
    x[9, :32] = np.float32(2.0 ** -126) * np.arange(32)
    x[10, :32] = np.float32(2.0 ** -121) * (1 - np.float32(2.0 ** -24)) * np.arange(32) / 31
    x[11] *= 1e30
    x[12] *= 1e-30
    x[13, :32] = np.nextafter(np.float32(2.0), np.float32(0))
    return torch.from_numpy(x)


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_rows8_bit_for_bit(ctx, dtype):
    x = special_rows().to(dtype)
    codes, exps, values = rows8(x)
    got = fs.fs_rows_pack8(ctx, x.cuda())
    assert np.array_equal(got.exps.cpu().numpy(), exps)
    assert np.array_equal(got.codes.cpu().numpy(), codes)
    back = fs.fs_rows_unpack8(ctx, got, dtype)
    assert back.dtype == dtype
    assert np.array_equal(back.cpu().double().numpy(), values, equal_nan=True)
    fine = np.isfinite(values)
    top = np.abs(np.where(fine, x.double().numpy(), 0)).reshape(40, 2, 32).max(-1).repeat(32, 1)
    off = np.where(fine, np.abs(values - np.where(fine, x.double().numpy(), 0)), 0)
    assert np.all(off <= np.maximum(top / 127, 2.0 ** -127))


@pytest.mark.parametrize("n,dim", [(1, 32), (3, 96), (64, 128), (1000, 160), (17, 1024), (50_001, 64)])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_rows8_sizes_and_strides(ctx, n, dim, dtype):
    x = rnd((n, dim), dtype, n)
    codes, exps, values = rows8(x)
    wide = torch.full((n, dim + 24), float("nan"), dtype=dtype, device="cuda")
    wide[:, 8:8 + dim] = x.cuda()
    for rows in (x.cuda(), wide[:, 8:8 + dim]):
        got = fs.fs_rows_pack8(ctx, rows)
        assert np.array_equal(got.codes.cpu().numpy(), codes) and np.array_equal(got.exps.cpu().numpy(), exps)
    out = torch.full_like(wide, -1.0)
    fs.fs_rows_unpack8(ctx, got, out=out[:, 8:8 + dim])
    assert np.array_equal(out[:, 8:8 + dim].cpu().double().numpy(), values)
    assert bool((out[:, :8] == -1).all()) and bool((out[:, 8 + dim:] == -1).all())


def test_every_code_and_exponent_reads_back(ctx):
    codes = torch.arange(-128, 128, dtype=torch.int16).to(torch.int8).repeat(256, 1).cuda()
    exps = torch.arange(256, dtype=torch.int16).to(torch.uint8).repeat_interleave(8).reshape(256, 8).cuda()
    got = fs.fs_rows_unpack8(ctx, fs.Rows8(codes, exps)).cpu().double()
    want = torch.arange(-128, 128, dtype=torch.float64) * torch.pow(2.0, torch.arange(256, dtype=torch.float64)[:, None] - 127)
    assert bool(got[255].isnan().all())
    assert torch.equal(got[:255], want[:255].float().double())


@pytest.mark.parametrize("n,dim,rows_dt,dt", [(1, 32, F32, F32), (333, 64, F32, BF16), (50, 160, BF16, BF16), (9, 1024, F32, BF16)])
def test_kept_in_8_bits_from_forward_to_backward(ctx, n, dim, rows_dt, dt):
    t = cuda(inputs(n, dim, rows_dt, dt))
    w = (t["w_post"], t["scale"], t["w_pre"])
    plain = fs.fs_block_norm(ctx, t["x"], t["a"], t["g"], *w, eps=EPS)
    got = fs.fs_block_norm(ctx, t["x"], t["a"], t["g"], *w, eps=EPS, pack=("a", "g", "y"))
    for k in ("y", "h"):
        assert torch.equal(got[k], plain[k])
    for k, rows in (("a8", t["a"]), ("g8", t["g"]), ("y8", plain["y"])):
        codes, exps, _ = rows8(rows)
        assert np.array_equal(got[k].codes.cpu().numpy(), codes) and np.array_equal(got[k].exps.cpu().numpy(), exps), k
    # the gradients are those at the values the codes stand for, whichever of the three are kept that way
    read = {k: fs.fs_rows_unpack8(ctx, got[k + "8"], rows_dt if k == "y" else dt) for k in ("a", "g", "y")}
    full = {"a": t["a"], "g": t["g"], "y": plain["y"]}
    for packed in ("a", "g", "y", "ag", "agy"):
        either = lambda k, p=packed: got[k + "8"] if k in p else full[k]  # noqa: E731
        same = lambda k, p=packed: read[k] if k in p else full[k]  # noqa: E731
        one = fs.fs_block_norm_backward(ctx, t["dy"], t["dh"], either("a"), either("g"), either("y"), *w, eps=EPS)
        two = fs.fs_block_norm_backward(ctx, t["dy"], t["dh"], same("a"), same("g"), same("y"), *w, eps=EPS)
        for k in two:
            assert torch.equal(one[k], two[k]), (packed, k)


# ---- how calls are made ----------------------------------------------------------------------------------------------------
def test_on_another_stream_and_twice_the_same(ctx):
    t = cuda(inputs(5000, 128, F32, BF16))
    w = (t["w_post"], t["scale"], t["w_pre"])
    y = fs.fs_block_norm(ctx, t["x"], t["a"], t["g"], *w, eps=EPS)["y"]
    want = fs.fs_block_norm_backward(ctx, t["dy"], t["dh"], t["a"], t["g"], y, *w, eps=EPS)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = [fs.fs_block_norm_backward(ctx, t["dy"], t["dh"], t["a"], t["g"], y, *w, eps=EPS, stream=s)
           for s in (side, None, side.cuda_stream, None)]
    torch.cuda.synchronize()
    for g in got:
        for k in want:
            assert torch.equal(g[k], want[k]), k


def test_captured_and_replayed(ctx):
    t = cuda(inputs(3000, 64, F32, BF16))
    w = (t["w_post"], t["scale"], t["w_pre"])

    def both():
        f = fs.fs_block_norm(ctx, t["x"], t["a"], t["g"], *w, eps=EPS, pack=("a", "g"))
        return {"h": f["h"], **fs.fs_block_norm_backward(ctx, t["dy"], t["dh"], f["a8"], f["g8"], f["y"], *w, eps=EPS, dtype=BF16)}

    both()
    torch.cuda.synchronize()
    graphs = []
    for _ in range(2):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            res = both()
        graphs.append((graph, res))
    for round_ in range(3):
        t["x"].copy_(rnd((3000, 64), F32, 100 + round_))
        t["dh"].copy_(rnd((3000, 64), BF16, 200 + round_))
        want = both()
        for graph, res in graphs:
            graph.replay()
        torch.cuda.synchronize()
        for graph, res in graphs:
            for k in want:
                assert torch.equal(res[k], want[k]), (round_, k)

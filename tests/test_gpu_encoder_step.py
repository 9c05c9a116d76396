"""One layer of a history encoder over an embedding table, made of the library's operators as a user has them together: lookup,
norm, attention with its position bias, gated join kept in 8 bits, the way back, and the updates of the table and of the bias;
against the same layer differentiated in 64 bits, and its form for one new row of each user against the training form."""
import numpy as np
import pytest
import torch

import oracle as O
import paper_2604_24073_amd as fs

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16
ROWS, DIM, HEADS, KV_HEADS, WIDTH, BUCKETS, DISTANCES, EPS = 500, 64, 4, 2, 32, 12, 90, 1e-6
LENS = [37, 0, 130, 1, 64, 200]
# Relative to a result's norm.  32 bits: six products follow one another, of up to 300 terms, whose roundings add up like the
# root of their number: 6 * 17 * 2^-24, and the powers of the softmax make up to ten times that of a score's error.  bf16: ten
# values on the way are rounded to 2^-9 of themselves (root mean square: 2^-9 / 1.7 each), both factors of a product at a time.
TOLERANCE = {F32: 6 * 17 * 10 * 2.0 ** -24, BF16: 2 * 10 * 2.0 ** -9}


@pytest.fixture(scope="module")
def ctx():
    c = fs.Context(max_ids=4096)
    yield c
    assert fs.fs_check_async(c) == fs.FS_OK, c.last_error()
    c.close()


def make(dtype, seed=0):
    gen = torch.Generator().manual_seed(seed)
    rnd = lambda *shape, size=1.0: torch.randn(shape, generator=gen) * size  # noqa: E731
    n, wide = sum(LENS), HEADS * WIDTH
    p = {"table": rnd(ROWS, DIM), "w_in": 1 + rnd(DIM, size=0.1), "w_post": 1 + rnd(DIM, size=0.1), "scale": 0.5 + rnd(DIM, size=0.1),
         "w_out": 1 + rnd(DIM, size=0.1), "bias": rnd(BUCKETS, HEADS, size=0.5),
         "qkv": rnd(DIM, (HEADS + 2 * KV_HEADS) * WIDTH, size=DIM ** -0.5).to(dtype), "gate": rnd(DIM, DIM, size=DIM ** -0.5).to(dtype),
         "back": rnd(wide, DIM, size=wide ** -0.5).to(dtype)}
    ids = torch.randint(0, ROWS, (n,), generator=gen)
    bucket_of = (torch.arange(DISTANCES).float().add(1).log2() * 2).clamp(max=BUCKETS - 1).to(torch.int32)
    offs = torch.tensor(np.concatenate([[0], np.cumsum(LENS)]), dtype=torch.int64)
    return p, ids, bucket_of, offs, rnd(n, DIM), rnd(n, DIM).to(dtype)


def layer(ctx, p, ids, bucket_of, offs, dy, dh, packed):
    """{name: result} of the forward and backward pass; p and the rest on the GPU."""
    dtype, n = dh.dtype, ids.numel()
    x = fs.fs_gather_jagged(ctx, p["table"], ids, offs)
    h = fs.fs_block_norm(ctx, x, w_pre=p["w_in"], eps=EPS, dtype=dtype)["h"]
    q, k, v = (h @ p["qkv"]).view(n, -1, WIDTH).split([HEADS, KV_HEADS, KV_HEADS], dim=1)
    position = {"bias": p["bias"], "bucket_of": bucket_of}
    kept = fs.fs_jagged_attention(ctx, q, k, v, offs, offs, **position, keep=True)
    a, g = kept["out"].flatten(1) @ p["back"], h @ p["gate"]
    weights = {"w_post": p["w_post"], "scale": p["scale"], "w_pre": p["w_out"], "eps": EPS}
    two = fs.fs_block_norm(ctx, x, a, g, **weights, pack=("a", "g") if packed else ())
    res = {"y": two["y"], "h": two["h"], "k": k, "v": v, "q": q, "out": kept["out"]}

    way = fs.fs_block_norm_backward(ctx, dy, dh, two["a8"] if packed else a, two["g8"] if packed else g, two["y"], **weights)
    plain = lambda name: fs.fs_rows_unpack8(ctx, two[name], dtype) if packed else {"a8": a, "g8": g}[name]  # noqa: E731
    same = fs.fs_block_norm_backward(ctx, dy, dh, plain("a8"), plain("g8"), two["y"], **weights)
    assert all(torch.equal(way[name], same[name]) for name in way)             # rows in 8 bits count as what they read back as
    dout = (way["da"] @ p["back"].t()).view_as(kept["out"])
    dqkv = torch.empty((n, HEADS + 2 * KV_HEADS, WIDTH), dtype=dtype, device="cuda")
    parts = dict(zip(("dq", "dk", "dv"), dqkv.split([HEADS, KV_HEADS, KV_HEADS], dim=1)))
    grads = fs.fs_jagged_attention_backward(ctx, dout, kept, q, k, v, offs, offs, **position, out=parts)
    inner = dqkv.flatten(1) @ p["qkv"].t() + way["dg"] @ p["gate"].t()
    first = fs.fs_block_norm_backward(ctx, way["dx"], inner, y=x, w_pre=p["w_in"], eps=EPS)
    res.update(dbias=grads["dbias"], drows=first["dx"], dw_in=first["dw_pre"], dw_post=way["dw_post"], dscale=way["dscale"],
               dw_out=way["dw_pre"])
    return res


def plain_layer(p, ids, bucket_of, dy, dh):
    """The same in 64 bits on the CPU, gradients by differentiation."""
    leaves = {n: t.double().requires_grad_() for n, t in p.items()}
    rms = lambda t: t / torch.sqrt((t * t).mean(1, keepdim=True) + EPS)  # noqa: E731
    x = leaves["table"][ids]
    x.retain_grad()
    h = rms(x) * leaves["w_in"]
    qkv = (h @ leaves["qkv"]).view(len(ids), -1, WIDTH)
    q, k, v = qkv.split([HEADS, KV_HEADS, KV_HEADS], dim=1)
    outs, at = [], 0
    for n in LENS:
        d = torch.arange(n)[:, None] - torch.arange(n)[None, :]
        bias = leaves["bias"][bucket_of[d.clamp(0, DISTANCES - 1)].long()].permute(2, 0, 1)
        kk, vv = (t[at:at + n].transpose(0, 1).repeat_interleave(HEADS // KV_HEADS, 0) for t in (k, v))
        s = q[at:at + n].transpose(0, 1) @ kk.transpose(1, 2) * WIDTH ** -0.5 + bias
        outs.append((torch.softmax(s.masked_fill(d < 0, -np.inf), 2) @ vv).transpose(0, 1))
        at += n
    out = torch.cat(outs)
    a, g = out.flatten(1) @ leaves["back"], h @ leaves["gate"]
    y = x + leaves["scale"] * leaves["w_post"] * rms(a) * torch.nn.functional.silu(g)
    h2 = rms(y) * leaves["w_out"]
    ((y * dy.double()).sum() + (h2 * dh.double()).sum()).backward()
    return {"y": y.detach(), "h": h2.detach(), "dbias": leaves["bias"].grad, "drows": x.grad, "dw_in": leaves["w_in"].grad,
            "dw_post": leaves["w_post"].grad, "dscale": leaves["scale"].grad, "dw_out": leaves["w_out"].grad}


@pytest.mark.parametrize("dtype,packed", [(F32, False), (BF16, False), (F32, True), (BF16, True)])
def test_a_layer_and_its_updates(ctx, dtype, packed):
    host, ids, bucket_of, offs, dy, dh = make(dtype)
    dev = {n: t.cuda() for n, t in host.items()}
    d_ids, d_buckets, d_offs = ids.cuda(), bucket_of.cuda(), offs.cuda()
    got, want = layer(ctx, dev, d_ids, d_buckets, d_offs, dy.cuda(), dh.cuda(), packed), plain_layer(host, ids, bucket_of, dy, dh)
    for name, w in want.items():
        off = float((got[name].cpu().double() - w).norm() / w.norm())
        # rows in 8 bits have steps of 2^-6 of their group's largest, which is up to three times the size of its values: off by
        # 2^-6 3 / sqrt(12) of themselves, and the gradients follow two of them
        assert off <= TOLERANCE[dtype] + (2 * 2.0 ** -6 if packed and name not in ("y", "h") else 0.0), (name, off)

    # the updates: the table's rows from the summed gradients of their occurrences, the bias as a table of its own
    lay = fs.fs_unique_ids(ctx, d_ids, ROWS)
    reduced = fs.fs_segment_reduce_grads(ctx, got["drows"], lay["perm"], lay["seg_offsets"], lay["n_unique"])
    u = int(lay["n_unique"])
    for table, rows, n_rows, sums, cap in (
            (dev["table"], lay["unique"], lay["n_unique"], reduced, u),
            (dev["bias"], torch.arange(BUCKETS, device="cuda"), torch.tensor([BUCKETS], device="cuda"), got["dbias"], BUCKETS)):
        t_ref, s_ref = table.cpu().numpy().copy(), np.zeros(len(table), np.float32)
        slots = torch.arange(cap, dtype=torch.int32)
        O.rowwise_adagrad_update(t_ref, s_ref, rows[:cap].cpu().numpy(), slots.numpy(), sums.cpu().numpy(), 0.05, 1e-8)
        state = torch.zeros(len(table), device="cuda")
        before = table.clone()
        fs.fs_rowwise_adagrad_update(ctx, table, state, rows, slots.cuda(), n_rows, cap, sums, 0.05, 1e-8)
        assert np.allclose(table.cpu().numpy(), t_ref, rtol=2.0 ** -20, atol=2.0 ** -22) and not torch.equal(table, before)
        assert np.allclose(state.cpu().numpy(), s_ref, rtol=2.0 ** -20)


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_one_new_row_of_each_user(ctx, dtype):
    """The last row of each history against a cache of the others: what the pass over whole histories had for it."""
    host, ids, bucket_of, offs, dy, dh = make(dtype, 1)
    dev = {n: t.cuda() for n, t in host.items()}
    d_buckets, d_offs = bucket_of.cuda(), offs.cuda()
    full = layer(ctx, dev, ids.cuda(), d_buckets, d_offs, dy.cuda(), dh.cuda(), False)
    users = [b for b, n in enumerate(LENS) if n]
    last = torch.tensor([int(offs[b]) + LENS[b] - 1 for b in users])
    x = fs.fs_gather_jagged(ctx, dev["table"], ids[last].cuda(), None)
    h = fs.fs_block_norm(ctx, x, w_pre=dev["w_in"], eps=EPS, dtype=dtype)["h"]
    new = (h @ dev["qkv"]).view(len(users), -1, WIDTH)
    room = 32
    k, v = (torch.full((sum(LENS) + room * len(LENS), KV_HEADS, WIDTH), float("nan"), dtype=dtype, device="cuda") for _ in range(2))
    starts = [int(offs[b]) + room * b for b in range(len(LENS))]
    for b, n in enumerate(LENS):
        for cache, name in ((k, "k"), (v, "v")):
            cache[starts[b]:starts[b] + n] = full[name][int(offs[b]):int(offs[b]) + n]
    for i, b in enumerate(users):
        k[starts[b] + LENS[b] - 1], v[starts[b] + LENS[b] - 1] = new[i, HEADS:HEADS + KV_HEADS], new[i, HEADS + KV_HEADS:]
    q_offs = torch.tensor(np.concatenate([[0], np.cumsum([min(n, 1) for n in LENS])]), dtype=torch.int64).cuda()
    kv_offs = torch.tensor(starts + [k.shape[0]], dtype=torch.int64).cuda()
    out = fs.fs_jagged_attention(ctx, new[:, :HEADS], k, v, q_offs, kv_offs, bias=dev["bias"], bucket_of=d_buckets,
                                 kv_lengths=torch.tensor(LENS).cuda(), max_q=1)["out"]
    two = fs.fs_block_norm(ctx, x, out.flatten(1) @ dev["back"], h @ dev["gate"], w_post=dev["w_post"], scale=dev["scale"],
                           w_pre=dev["w_out"], eps=EPS)
    for name in ("y", "h"):
        want = full[name][last.cuda()].double()
        assert float((two[name].double() - want).norm() / want.norm()) <= 2 * TOLERANCE[dtype], name

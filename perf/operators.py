"""The operators of a history encoder, as cases that can be timed: jagged attention with a learned relative position
bias, the norms around a block with its gate and residual scale, and rows held in 8 bits.

A case is a dict of plain values.  `listed()` names twelve of them, `draw(rng)` makes more over the same ranges, `prepare`
builds what a program holds before the call, `run` is one pass, either through the plain forms below (elementary torch
operations in 32 bits, `own` false) or through the library's entry points (`own` true), `exact` computes the same from the
definitions in 64 bits, and `work` counts the bytes and operations that no implementation can avoid.

Kinds of passes
  attend    attention over a jagged batch, forward and backward: out, dq, dk, dv and the bias table's gradient
  serve     attention of a few new rows of each user over the user's cached history, which has rows to spare
  join      y = x + scale * w_post * rms(a) * silu(g), h = w_pre * rms(y): forward, and backward where `train`; `packed`: the
            backward pass reads a and g as the forward pass left them in 8 bits
  rows8     rows to 8 bits and back

Lengths are the quantiles of their distribution at evenly spaced points, shuffled by the seed: a case has the same size
whatever the seed.
"""
import math

import numpy as np
import torch

own = False

LONG_HISTORY = 16_384           # the 5 % long histories of the skewed batches
EPS = 1e-6
GROUP = 32                      # columns that share a power of two in 8 bits
NEG = float("-inf")


# ---- the cases -------------------------------------------------------------------------------------------------
def _attend(users, rule, lo, hi, heads, kv_heads, head_dim, dtype, buckets, distances, causal=True):
    return {"kind": "attend", "users": users, "lengths": rule, "lo": lo, "hi": hi, "heads": heads, "kv_heads": kv_heads,
            "head_dim": head_dim, "dtype": dtype, "buckets": buckets, "distances": distances, "causal": causal}


def _serve(users, lo, hi, rows, heads, kv_heads, head_dim, dtype, buckets, distances):
    return {"kind": "serve", "users": users, "lengths": "powerlaw", "lo": lo, "hi": hi, "rows": rows, "heads": heads,
            "kv_heads": kv_heads, "head_dim": head_dim, "dtype": dtype, "buckets": buckets, "distances": distances,
            "causal": True}


def _join(n, dim, rows, dtype, train, packed=False):
    return {"kind": "join", "n": n, "dim": dim, "rows": rows, "dtype": dtype, "train": train, "packed": packed}


def listed():
    return [
        # the smallest training batch there is, all latency
        {"name": "attend_tiny", **_attend(32, "uniform", 1, 64, 2, 2, 32, "f32", 32, 64)},
        # a training batch of one shard, rows of 128 columns in four heads
        {"name": "attend_shard", **_attend(1024, "powerlaw", 16, 4096, 4, 4, 32, "bf16", 64, 2048)},
        # a few users with very long histories, heads in groups: the largest pass
        {"name": "attend_long", **_attend(160, "skew", 8, 256, 4, 2, 64, "bf16", 64, 4096)},
        # an encoder that looks both ways, odd lengths and an odd width of its heads, in 32 bits
        {"name": "attend_both_ways", **_attend(77, "powerlaw", 1, 777, 3, 3, 40, "f32", 33, 129, causal=False)},
        # one new event of each of 256 users against the cached history
        {"name": "serve_token", **_serve(256, 16, 8192, 1, 8, 2, 64, "bf16", 64, 2048)},
        # a handful of users with short histories, four new events each, all latency
        {"name": "serve_few", **_serve(5, 1, 300, 4, 4, 4, 32, "f32", 32, 64)},
        # between two blocks of the smallest training batch
        {"name": "join_tiny", **_join(927, 64, "f32", "f32", True)},
        # between two blocks of a shard's batch, residual rows in 32 bits, the block's in 16
        {"name": "join_shard", **_join(297_000, 128, "f32", "bf16", True)},
        # wide rows, the block's output and gate kept in 8 bits from forward to backward
        {"name": "join_packed", **_join(200_003, 256, "f32", "bf16", True, True)},
        # the same place in serving: one row of each user, no gradients
        {"name": "join_serve", **_join(256, 512, "bf16", "bf16", False)},
        # the gathered rows of a shard's batch kept in 8 bits
        {"name": "rows8_shard", "kind": "rows8", "n": 297_000, "dim": 128, "dtype": "f32"},
        # those of the smallest batch
        {"name": "rows8_tiny", "kind": "rows8", "n": 927, "dim": 64, "dtype": "bf16"},
    ]


def _log_between(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _pairs(lens):
    return float((np.asarray(lens, np.float64) ** 2).sum())


def draw(rng):
    kind = rng.choice(["attend", "attend", "serve", "join", "join", "rows8"])
    dtype = rng.choice(["f32", "bf16", "bf16"])
    if kind == "rows8":
        return {"kind": kind, "n": _log_between(rng, 1, 297_000), "dim": GROUP * rng.randint(1, 4), "dtype": dtype}
    if kind == "join":
        n = _log_between(rng, 1, 200_000)
        dim = GROUP * rng.randint(1, 16) if n < 50_000 else GROUP * rng.randint(1, 8)
        if rng.random() < 0.3:
            return _join(n, dim, rng.choice(["f32", dtype]), dtype, False)
        if rng.random() < 0.5:
            return _join(n, dim, "f32", dtype, True, True)
        return _join(n, max(8, dim - 8 * rng.randint(0, 3)), "f32", dtype, True)
    kv_heads = rng.choice([1, 2, 3, 4])
    heads = kv_heads * rng.choice([1, 1, 2, 4])
    head_dim = rng.choice([32, 64, 128, 8 * rng.randint(1, 16)])
    buckets, distances = rng.randint(1, 128), _log_between(rng, 1, 4096)
    if kind == "serve":
        rows = rng.choice([1, 1, 1, 2, 3, 4])
        return _serve(_log_between(rng, 1, 256), _log_between(rng, 1, 64), _log_between(rng, 65, 8192), rows, heads, kv_heads,
                      head_dim, dtype, buckets, distances)
    case = _attend(_log_between(rng, 1, 512), rng.choice(["uniform", "powerlaw"]), _log_between(rng, 1, 16),
                   _log_between(rng, 17, 4096), heads, kv_heads, head_dim, dtype, buckets, distances, rng.random() < 0.75)
    most = 1.5e9 if dtype == "bf16" else 1.5e8          # pairs of rows times heads
    while _pairs(_lengths(case)) * heads > most and (case["hi"] > 2 * case["lo"] + 1 or case["users"] > 1):
        if case["hi"] > 2 * case["lo"] + 1:
            case["hi"] = max(2 * case["lo"] + 1, case["hi"] * 3 // 4)
        case["users"] = max(1, case["users"] * 3 // 4)
    return case


# ---- inputs ----------------------------------------------------------------------------------------------------
def _lengths(case):
    """int64 [users], ascending: quantiles of the length rule."""
    n, lo, hi = case["users"], case["lo"], case["hi"]
    q = (np.arange(n) + 0.5) / n
    if case["lengths"] == "powerlaw":               # density x^-1.5 on [lo, hi + 1)
        a, b = lo ** -0.5, (hi + 1) ** -0.5
        x = (a + q * (b - a)) ** -2.0
    else:
        x = lo + q * (hi + 1 - lo)
    lens = np.clip(np.floor(x).astype(np.int64), lo, hi)
    if case["lengths"] == "skew":                   # 5 % of the users have a very long history
        long = max(1, round(0.05 * n))
        lens = np.concatenate([lens[:n - long], np.full(long, LONG_HISTORY, np.int64)])
    return lens


def _dtype(name):
    return torch.float32 if name == "f32" else torch.bfloat16


def _normal(gen, shape, dtype=torch.float32, size=1.0):
    return (torch.randn(shape, dtype=torch.float32, device="cuda", generator=gen) * size).to(dtype)


def _offsets(lens):
    return np.concatenate([[0], np.cumsum(lens)]).astype(np.int64)


def _bucket_table(buckets, distances, causal):
    """Bucket of each distance, exact up to half of the buckets and logarithmic behind; where both directions count, the
    first half of the buckets is for rows behind and the second for rows ahead."""
    per = buckets if causal else max(1, buckets // 2)
    d = np.arange(distances)
    near = max(1, per // 2)
    far = near + np.log(np.maximum(d, near) / near) / max(math.log(max(distances, near + 1) / near), 1e-9) * (per - near)
    b = np.where(d < near, d, np.minimum(far.astype(np.int64), per - 1))
    b = np.minimum(b, per - 1)
    if not causal:
        b = np.concatenate([np.minimum(b[:0:-1] + per, buckets - 1), b])
    return b.astype(np.int32)


def _context():
    import paper_2604_24073_amd as fs
    if "ctx" not in _held:
        _held["ctx"] = fs.Context(max_ids=4096)
    return _held["ctx"]


_held = {}                      # the one context of the process, as a program holds it


def prepare(case, seed):
    rng = np.random.default_rng(seed)
    gen = torch.Generator(device="cuda").manual_seed(seed)
    state = {"case": case}
    if own:
        state["ctx"] = _context()
    if case["kind"] == "rows8":
        state["rows"] = _normal(gen, (case["n"], case["dim"]), _dtype(case["dtype"]))
        return state
    if case["kind"] == "join":
        n, dim, dtype = case["n"], case["dim"], _dtype(case["dtype"])
        state["x"] = _normal(gen, (n, dim), _dtype(case["rows"]))
        state["a"], state["g"] = _normal(gen, (n, dim), dtype, 0.7), _normal(gen, (n, dim), dtype)
        for name, mid in (("w_post", 1.0), ("scale", 0.5), ("w_pre", 1.0)):
            state[name] = mid + _normal(gen, (dim,), size=0.1)
        if case["train"]:
            state["dy"], state["dh"] = _normal(gen, (n, dim), _dtype(case["rows"])), _normal(gen, (n, dim), dtype)
        return state
    heads, kv_heads, hd, dtype = case["heads"], case["kv_heads"], case["head_dim"], _dtype(case["dtype"])
    lens = rng.permutation(_lengths(case))
    state["bias"] = _normal(gen, (case["buckets"], heads), size=0.5)
    state["bucket_of"] = torch.from_numpy(_bucket_table(case["buckets"], case["distances"], case["causal"])).cuda()
    if case["kind"] == "attend":
        offs = _offsets(lens)
        n = int(offs[-1])
        state["host"] = (offs, offs, lens)
        state["kv_offsets"] = state["q_offsets"] = torch.from_numpy(offs).cuda()
        # one projection makes the three of them, so that their rows lie in one tensor
        qkv = _normal(gen, (n, heads + 2 * kv_heads, hd), dtype)
        state["q"], state["k"], state["v"] = qkv.split([heads, kv_heads, kv_heads], dim=1)
        state["dout"] = _normal(gen, (n, heads, hd), dtype)
        return state
    room = (lens + 127) // 64 * 64                     # what the cache holds for each user
    offs, q_offs = _offsets(room), _offsets(np.full(len(lens), case["rows"]))
    state["host"] = (q_offs, offs, lens)
    state["q_offsets"], state["kv_offsets"] = torch.from_numpy(q_offs).cuda(), torch.from_numpy(offs).cuda()
    state["kv_lengths"] = torch.from_numpy(np.ascontiguousarray(lens)).cuda()
    state["q"] = _normal(gen, (int(q_offs[-1]), heads, hd), dtype)
    state["k"], state["v"] = _normal(gen, (int(offs[-1]), kv_heads, hd), dtype), _normal(gen, (int(offs[-1]), kv_heads, hd), dtype)
    return state


# ---- plain forms -----------------------------------------------------------------------------------------------
def _visible(state, b, causal, device):
    """(index into the bucket table [rows, keys], who sees whom) of user b: the rows are the last ones of the history."""
    q_offs, _, lens = state["host"]
    rows, keys = int(q_offs[b + 1] - q_offs[b]), int(lens[b])
    d = (torch.arange(rows, device=device) + (keys - rows))[:, None] - torch.arange(keys, device=device)[None, :]
    size = state["bucket_of"].numel()
    if causal:
        return d.clamp(0, size - 1), d >= 0
    mid = size // 2
    return d.clamp(-mid, mid) + mid, None


def _plain_attention(state, train):
    case = state["case"]
    heads, kv_heads, hd, causal = case["heads"], case["kv_heads"], case["head_dim"], case["causal"]
    q, k, v, bias = state["q"], state["k"], state["v"], state["bias"]
    group, scale = heads // kv_heads, 1.0 / math.sqrt(hd)
    out = torch.zeros((q.shape[0], heads, hd), dtype=torch.float32, device=q.device)
    if train:
        dq, dk, dv = torch.zeros_like(out), *(torch.zeros((k.shape[0], kv_heads, hd), device=q.device) for _ in range(2))
        dbias = torch.zeros(bias.shape, dtype=torch.float64, device=q.device)
    q_offs, offs, lens = state["host"]
    for b in range(case["users"]):
        rq, rk = slice(int(q_offs[b]), int(q_offs[b + 1])), slice(int(offs[b]), int(offs[b] + lens[b]))
        index, seen = _visible(state, b, causal, q.device)
        bucket = state["bucket_of"][index].long()
        # [heads that share keys, heads that read them, rows, columns]
        kk, vv = (t[rk].float().transpose(0, 1)[:, None] for t in (k, v))
        qq = q[rq].float().transpose(0, 1).unflatten(0, (kv_heads, group))
        s = torch.matmul(qq, kk.transpose(2, 3)) * scale
        s += bias.t()[:, bucket].unflatten(0, (kv_heads, group))
        if seen is not None:
            s.masked_fill_(~seen, NEG)
        top = s.amax(-1, keepdim=True)
        p = torch.exp(s - torch.where(top == NEG, torch.zeros_like(top), top))
        del s
        total = p.sum(-1, keepdim=True)
        p /= torch.where(total > 0, total, torch.ones_like(total))
        o = torch.matmul(p, vv)
        out[rq] = o.flatten(0, 1).transpose(0, 1)
        if not train:
            continue
        do = state["dout"][rq].float().transpose(0, 1).unflatten(0, (kv_heads, group))
        dv[rk] = torch.matmul(p.transpose(2, 3), do).sum(1).transpose(0, 1)
        ds = torch.matmul(do, vv.transpose(2, 3))
        ds -= (do * o).sum(-1, keepdim=True)
        ds *= p
        del p
        dq[rq] = (torch.matmul(ds, kk) * scale).flatten(0, 1).transpose(0, 1)
        dk[rk] = (torch.matmul(ds.transpose(2, 3), qq).sum(1) * scale).transpose(0, 1)
        # a bucket's share of a distance: every row one column further right than the row above it, then the sums of
        # the columns; in 64 bits, for a bucket takes in millions of terms that nearly cancel
        rows, keys = ds.shape[2:]
        flat = torch.nn.functional.pad(ds.flatten(0, 1).flip(2), (0, rows)).reshape(heads, -1)[:, :rows * (keys + rows - 1)]
        del ds
        line = flat.reshape(heads, rows, keys + rows - 1).sum(1, dtype=torch.float64)
        far = state["bucket_of"].numel() // 2 if seen is None else 0
        d = torch.arange(keys + rows - 1, device=q.device) - (rows - 1) + far
        dbias.index_add_(0, state["bucket_of"][d.clamp(0, state["bucket_of"].numel() - 1)].long(), line.t())
        del flat
    if not train:
        return {"out": out.to(q.dtype)}
    return {"out": out.to(q.dtype), "dq": dq.to(q.dtype), "dk": dk.to(q.dtype), "dv": dv.to(q.dtype), "dbias": dbias.float()}


def _plain_codes(rows):
    """(codes, power of two) of each group of columns, as 32-bit values."""
    x = rows.float().reshape(rows.shape[0], -1, GROUP)
    top = x.abs().amax(-1, keepdim=True)
    e = (torch.frexp(top)[1] - 7).clamp(min=-126)
    e = torch.where(torch.ldexp(top, -e) >= 127.5, e + 1, e)
    step = torch.ldexp(torch.ones_like(top), e)
    return torch.round(x / step), step


def _plain_rows8(rows):
    codes, step = _plain_codes(rows)
    return (codes * step).reshape(rows.shape).to(rows.dtype)


def _plain_rms(x):
    r = torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS)
    return x * r, r


def _plain_rms_grad(dxhat, xhat, r):
    return r * (dxhat - xhat * (dxhat * xhat).mean(-1, keepdim=True))


def _plain_join(state):
    case, x, a, g = state["case"], state["x"], state["a"], state["g"]
    w_post, scale, w_pre = state["w_post"], state["scale"], state["w_pre"]
    ahat, _ = _plain_rms(a.float())
    gate = torch.sigmoid(g.float())
    y = x.float() + scale * w_post * ahat * (g.float() * gate)
    yhat, ry = _plain_rms(y)
    res = {"y": y.to(x.dtype), "h": (yhat * w_pre).to(a.dtype)}
    if not case["train"]:
        return res
    af, gf = (_plain_rows8(t).float() if case["packed"] else t.float() for t in (a, g))
    ahat, ra = _plain_rms(af)
    gate = torch.sigmoid(gf)
    dh = state["dh"].float()
    dx = state["dy"].float() + _plain_rms_grad(dh * w_pre, yhat, ry)
    t = dx * (scale * w_post)
    res["dx"] = dx.to(x.dtype)
    res["da"] = _plain_rms_grad(t * (gf * gate), ahat, ra).to(a.dtype)
    res["dg"] = (t * ahat * (gate * (1 + gf * (1 - gate)))).to(a.dtype)
    both = (dx * (gf * gate) * ahat).double().sum(0)             # long sums
    res["dw_post"], res["dscale"] = (both * scale).float(), (both * w_post).float()
    res["dw_pre"] = (dh * yhat).double().sum(0).float()
    return res


# ---- the library's calls ---------------------------------------------------------------------------------------
def _own_attention(state, train):
    import paper_2604_24073_amd as fs
    case, ctx = state["case"], state["ctx"]
    what = dict(bias=state["bias"], bucket_of=state["bucket_of"], causal=case["causal"])
    args = (state["q"], state["k"], state["v"], state["q_offsets"], state["kv_offsets"])
    if not train:
        res = fs.fs_jagged_attention(ctx, *args, kv_lengths=state["kv_lengths"], max_q=case["rows"], **what)
        return {"out": res["out"]}
    kept = fs.fs_jagged_attention(ctx, *args, keep=True, **what)
    res = fs.fs_jagged_attention_backward(ctx, state["dout"], kept, *args, **what)
    return {"out": kept["out"], **{k: res[k] for k in ("dq", "dk", "dv", "dbias")}}


def _own_join(state):
    import paper_2604_24073_amd as fs
    case, ctx = state["case"], state["ctx"]
    weights = (state["w_post"], state["scale"], state["w_pre"])
    res = fs.fs_block_norm(ctx, state["x"], state["a"], state["g"], *weights, eps=EPS, pack=("a", "g") if case["packed"] else ())
    ret = {"y": res["y"], "h": res["h"]}
    if case["train"]:
        a, g = (res["a8"], res["g8"]) if case["packed"] else (state["a"], state["g"])
        ret.update(fs.fs_block_norm_backward(ctx, state["dy"], state["dh"], a, g, res["y"], *weights, eps=EPS,
                                             dtype=state["a"].dtype))
    return {k: ret[k] for k in (JOINED if case["train"] else JOINED[:2])}


JOINED = ("y", "h", "dx", "da", "dg", "dw_post", "dscale", "dw_pre")


def run(state):
    case = state["case"]
    if case["kind"] == "rows8":
        if not own:
            return _plain_rows8(state["rows"])
        import paper_2604_24073_amd as fs
        packed = fs.fs_rows_pack8(state["ctx"], state["rows"])
        return fs.fs_rows_unpack8(state["ctx"], packed, state["rows"].dtype)
    if case["kind"] == "join":
        return _own_join(state) if own else _plain_join(state)
    return (_own_attention if own else _plain_attention)(state, case["kind"] == "attend")


# ---- from the definitions, in 64 bits ----------------------------------------------------------------------------
def _exact_attention(case, state, train):
    """Softmax by logsumexp, gradients by differentiation, one user and head at a time."""
    heads, group, hd = case["heads"], case["heads"] // case["kv_heads"], case["head_dim"]
    leaves = {n: state[n].detach().double().requires_grad_(train) for n in ("q", "k", "v")}
    bias = state["bias"].double()
    dbias = torch.zeros_like(bias)
    out = torch.zeros(leaves["q"].shape, dtype=torch.float64, device="cuda")
    q_offs, offs, lens = state["host"]
    table = state["bucket_of"].long()
    for b in range(case["users"]):
        rows, keys = int(q_offs[b + 1] - q_offs[b]), int(lens[b])
        i = torch.arange(keys - rows, keys, device="cuda").reshape(-1, 1)
        j = torch.arange(keys, device="cuda").reshape(1, -1)
        far = table.numel() - 1 if case["causal"] else (table.numel() - 1) // 2
        bucket = table[torch.minimum((i - j).clamp(min=0), torch.tensor(far, device="cuda"))] if case["causal"] else \
            table[far + torch.sign(i - j) * torch.minimum((i - j).abs(), torch.tensor(far, device="cuda"))]
        hidden = (j > i) if case["causal"] else torch.zeros_like(bucket, dtype=torch.bool)
        none = hidden.all(1, keepdim=True)
        for h in range(heads):
            q = leaves["q"][q_offs[b]:q_offs[b + 1], h]
            k, v = (leaves[n][offs[b]:offs[b] + keys, h // group] for n in ("k", "v"))
            s = (q @ k.T) / hd ** 0.5 + bias[:, h][bucket]
            if train:
                s.retain_grad()
            raw, s = s, s.masked_fill(hidden & ~none, NEG)
            o = torch.where(none, 0.0, 1.0) * (torch.exp(s - torch.logsumexp(s, 1, keepdim=True)) @ v)
            out[q_offs[b]:q_offs[b + 1], h] = o.detach()
            if not train:
                continue
            o.backward(state["dout"][q_offs[b]:q_offs[b + 1], h].double())
            if raw.numel() < 1 << 20:
                dbias[:, h].index_add_(0, bucket.reshape(-1), raw.grad.reshape(-1))
            else:
                for c in range(case["buckets"]):
                    dbias[c, h] += torch.where(bucket == c, raw.grad, 0.0).sum()
    if not train:
        return {"out": out}
    return {"out": out, "dq": leaves["q"].grad, "dk": leaves["k"].grad, "dv": leaves["v"].grad, "dbias": dbias}


def _exact_rows8(rows):
    x = rows.double().cpu().numpy().reshape(rows.shape[0], -1, GROUP)
    top = np.abs(x).max(-1, keepdims=True)
    e = np.maximum(np.floor(np.log2(np.where(top > 0, top, 1.0))) - 6, -126)
    e = e + (np.rint(top / 2.0 ** e) > 127)
    return torch.from_numpy((np.rint(x / 2.0 ** e) * 2.0 ** e).reshape(rows.shape)).cuda()


def _exact_join(case, state):
    leaf = lambda t: t.detach().double().requires_grad_(True)  # noqa: E731
    w_post, scale, w_pre = (leaf(state[n]) for n in ("w_post", "scale", "w_pre"))

    def norm(t):
        return t / torch.sqrt(t.square().sum(1, keepdim=True) / t.shape[1] + EPS)

    def joined(x, a, g):
        return x + scale * (w_post * norm(a)) * (g / (1 + torch.exp(-g)))

    x, a, g = (leaf(state[n]) for n in ("x", "a", "g"))
    y = joined(x, a, g)
    h = w_pre * norm(y)
    res = {"y": y.detach(), "h": h.detach()}
    if not case["train"]:
        return res
    # the path behind y is differentiated at the true y, what is in front of it at the rows that were kept
    mid = leaf(y)
    (w_pre * norm(mid)).backward(state["dh"].double())
    dx = state["dy"].double() + mid.grad
    a, g = (leaf(_exact_rows8(state[n]) if case["packed"] else state[n]) for n in ("a", "g"))
    joined(x.detach(), a, g).backward(dx)
    return {**res, "dx": dx, "da": a.grad, "dg": g.grad, "dw_post": w_post.grad, "dscale": scale.grad, "dw_pre": w_pre.grad}


def exact(case, seed):
    global own
    was, own = own, False
    try:
        state = prepare(case, seed)
    finally:
        own = was
    if case["kind"] == "rows8":
        return _exact_rows8(state["rows"])
    if case["kind"] == "join":
        return _exact_join(case, state)
    return _exact_attention(case, state, case["kind"] == "attend")


# ---- what a pass cannot do without -----------------------------------------------------------------------------
def work(case):
    size = 4 if case["dtype"] == "f32" else 2
    if case["kind"] == "rows8":
        n = case["n"] * case["dim"]
        return {"bytes": 2 * size * n, "flops": 4 * n}
    if case["kind"] == "join":
        n, row = case["n"] * case["dim"], 4 if case["rows"] == "f32" else 2
        # x, a, g in and y, h out; dy, dh in and dx, da, dg out
        return {"bytes": n * (2 * row + 3 * size + (2 * row + 3 * size if case["train"] else 0)),
                "flops": n * (50 if case["train"] else 15)}
    lens = _lengths(case)
    heads, kv_heads, hd = case["heads"], case["kv_heads"], case["head_dim"]
    if case["kind"] == "serve":
        rows = case["rows"]
        n = np.maximum(lens[:, None] - rows + 1 + np.arange(rows)[None, :], 0).clip(max=lens[:, None])
        return {"bytes": size * hd * (2 * rows * len(lens) * heads + 2 * int(lens.sum()) * kv_heads),
                "flops": 4 * hd * heads * int(n.sum())}
    pairs = int((lens * (lens + 1) // 2).sum()) if case["causal"] else int((lens * lens).sum())
    # q, k, v, dout in and out, dq, dk, dv out
    return {"bytes": size * hd * int(lens.sum()) * (4 * heads + 4 * kv_heads), "flops": 14 * hd * heads * pairs}

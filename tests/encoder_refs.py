"""The history encoder's operators from their definitions, in 64 bits on the CPU, each value with the sum of the magnitudes it
is made of: that is what the roundings of a 32-bit computation are relative to."""
import numpy as np
import torch

U32 = 2.0 ** -24                 # half a step of fp32, relative


def half_step(dtype):
    return torch.finfo(dtype).eps / 2


def assert_within(got, want, magnitude, roundings, what=""):
    """|got - want| <= half a step of got's type, and so many roundings in 32 bits of the magnitudes that went in."""
    got64 = got.detach().cpu().double()
    tol = half_step(got.dtype) * want.abs() + roundings * U32 * magnitude + 1e-37
    bad = ~((got64 - want).abs() <= tol) & ~(got64.isnan() & want.isnan()) & ~(got64 == want)
    if bool(bad.any()):
        k = int(bad.flatten().nonzero()[0])
        raise AssertionError(f"{what}: {int(bad.sum())} of {bad.numel()} beyond their bound, first at {k}: "
                             f"{got64.flatten()[k].item()} against {want.flatten()[k].item()}, bound {tol.flatten()[k].item()}")


def rows8(x):
    """(codes, exponent bytes, values) as numpy arrays; a group with a value that is no number reads NaN."""
    x = np.asarray(x.double().cpu() if isinstance(x, torch.Tensor) else x, np.float64)
    n, dim = x.shape
    g = x.reshape(n, dim // 32, 32)
    fine = np.isfinite(g).all(-1)
    g = np.where(fine[..., None], g, 0.0)
    top = np.abs(g).max(-1)
    e = np.where(top > 0, np.floor(np.log2(np.where(top > 0, top, 1.0))), -1000.0)
    # log2 of the value just below a power of two may round up to it
    e = np.where((top > 0) & (np.ldexp(1.0, e.astype(int)) > top), e - 1, e)
    e = np.maximum(e - 6, -126).astype(int)
    e = np.minimum(e + (np.rint(top / np.ldexp(1.0, e)) > 127), 121)
    codes = np.rint(g / np.ldexp(1.0, e)[..., None]).clip(-127, 127)
    values = np.where(fine[..., None], codes * np.ldexp(1.0, e)[..., None], np.nan)
    return codes.reshape(n, dim).astype(np.int8), np.where(fine, e + 127, 255).astype(np.uint8), values.reshape(n, dim)


def _rms(t, eps):
    r = 1 / torch.sqrt((t * t).mean(1, keepdim=True) + eps)
    return t * r, r


def block_norm(x, a, g, w_post, scale, w_pre, eps):
    """{name: (value, magnitude)} of y and h."""
    y, m = x, x.abs()
    if a is not None:
        ahat, _ = _rms(a, eps)
        term = scale * w_post * ahat * (g * torch.sigmoid(g))
        y, m = x + term, x.abs() + term.abs() * (1 + g.abs())          # exp(-g) is as good as its argument
    res = {"y": (y, m)}
    if w_pre is not None:
        yhat, r = _rms(y, eps)
        ym = m * r
        res["h"] = (yhat * w_pre, (ym + yhat.abs() * (ym * yhat.abs()).mean(1, keepdim=True)) * w_pre.abs())
    return res


def block_norm_backward(dy, dh, a, g, y, w_post, scale, w_pre, eps):
    res = {}
    dx = torch.zeros_like(y) if dy is None else dy
    dxm = dx.abs()
    if dh is not None:
        yhat, r = _rms(y, eps)
        u = dh * w_pre
        dx = dx + r * (u - yhat * (u * yhat).mean(1, keepdim=True))
        dxm = dxm + r * (u.abs() + yhat.abs() * (u * yhat).abs().mean(1, keepdim=True))
        res["dw_pre"] = ((dh * yhat).sum(0), (dh * yhat).abs().sum(0))
    res["dx"] = (dx, dxm)
    if a is not None:
        ahat, r = _rms(a, eps)
        gate = torch.sigmoid(g)
        silu = g * gate
        u, um = dx * scale * w_post, dxm * (scale * w_post).abs() * (1 + g.abs())
        res["dg"] = (u * ahat * gate * (1 + g * (1 - gate)), um * ahat.abs() * gate * (1 + g.abs() * (1 - gate)))
        res["da"] = (r * (u * silu - ahat * (u * silu * ahat).mean(1, keepdim=True)),
                     r * (um * silu.abs() + ahat.abs() * (um * silu * ahat).abs().mean(1, keepdim=True)))
        t, tm = (dx * ahat * silu).sum(0), (dxm * (1 + g.abs()) * (ahat * silu).abs()).sum(0)
        res["dw_post"], res["dscale"] = (t * scale, tm * scale.abs()), (t * w_post, tm * w_post.abs())
    return res


# ---- attention -------------------------------------------------------------------------------------------------------------
def attention(q, k, v, q_lens, k_lens, k_rooms, bias, bucket_of, causal, scale, dtype, dout=None):
    """{name: (value, error bound before the last rounding)} of out and lse, and with dout of the gradients.  All tensors in 64
    bits; user after user, head after head.  u is a 32-bit rounding, t one to the type of the rows (P and dS go into their
    products in it)."""
    u, t = U32, half_step(dtype) if dtype != torch.float32 else 0.0
    heads, width, group = q.shape[1], q.shape[2], q.shape[1] // k.shape[1]
    z = lambda like: torch.zeros_like(like)  # noqa: E731
    out, out_e, lse, lse_e = z(q), z(q), torch.full((heads, q.shape[0]), -np.inf, dtype=torch.float64), z(q[:, :, 0].t())
    grads = {n: [z(x), z(x)] for n, x in (("dq", q), ("dk", k), ("dv", v))}
    if bias is not None:
        grads["dbias"] = [z(bias), z(bias)]
    qa = ka = 0
    for nq, nk, room in zip(q_lens, k_lens, k_rooms):
        pos = torch.arange(nq)[:, None] + (nk - nq)
        d = pos - torch.arange(nk)[None, :]
        seen = d >= 0 if causal else torch.ones_like(d, dtype=torch.bool)
        if bias is not None:
            size = len(bucket_of)
            bucket = bucket_of[d.clamp(0, size - 1) if causal else d.clamp(-(size // 2), size // 2) + size // 2].long()
        for h in range(heads if nq and nk else 0):
            qh, kh, vh = q[qa:qa + nq, h], k[ka:ka + nk, h // group], v[ka:ka + nk, h // group]
            s = scale * (qh @ kh.T)
            mag = abs(scale) * (qh.abs() @ kh.abs().T)
            if bias is not None:
                b = bias[:, h][bucket]
                s, mag = s + b, mag + torch.where(b.isinf(), 0.0, b.abs())
            sees = seen & (s > -np.inf)
            s = s.masked_fill(~seen, -np.inf)
            L = torch.logsumexp(s, 1, keepdim=True)
            none = ~sees.any(1, keepdim=True)
            p = torch.where(none, 0.0, torch.exp(s - torch.where(none, 0.0, L)))
            # a score's error: its product's terms one after the other, scaling and bias, and the power's own
            es = torch.where(sees, (width + 8) * u * mag, 0.0)
            es = torch.where(sees.any(1, keepdim=True), es.amax(1, keepdim=True), 0.0)
            ep = 2 * es + (nk + 64) * u + 4 * u * torch.where(none, 0.0, L.abs())
            o, oe = p @ vh, (ep + t) * (p @ vh.abs())
            out[qa:qa + nq, h], out_e[qa:qa + nq, h] = o, oe
            lse[h, qa:qa + nq], lse_e[h, qa:qa + nq] = L[:, 0], (es + (nk + 64) * u + 4 * u * torch.where(none, 0.0, L.abs()))[:, 0]
            if dout is None:
                continue
            do = dout[qa:qa + nq, h]
            dp, dpm = do @ vh.T, do.abs() @ vh.abs().T
            D, Dm = (do * o).sum(1, keepdim=True), (do * o).abs().sum(1, keepdim=True)
            ds = p * (dp - D)
            # D is made of the unrounded out, whose error is that of P in its product
            De = width * u * Dm + (do.abs() * oe).sum(1, keepdim=True)
            dse = p * (width * u * dpm + De + (ep + 4 * u) * (dp - D).abs())
            into = dse + (t + (nk + 8) * u) * ds.abs()
            grads["dq"][0][qa:qa + nq, h] += scale * (ds @ kh)
            grads["dq"][1][qa:qa + nq, h] += abs(scale) * (into @ kh.abs())
            into = dse + (t + (nq * group + 8) * u) * ds.abs()
            grads["dk"][0][ka:ka + nk, h // group] += scale * (ds.T @ qh)
            grads["dk"][1][ka:ka + nk, h // group] += abs(scale) * (into.T @ qh.abs())
            grads["dv"][0][ka:ka + nk, h // group] += p.T @ do
            grads["dv"][1][ka:ka + nk, h // group] += ((ep + t + (nq * group + 8) * u) * p).T @ do.abs()
            if bias is not None:
                # 16 x 64 values of a wavefront, tile after tile, then in 64 bits
                one = dse + (1024 + nk) * u * ds.abs()
                grads["dbias"][0][:, h].index_add_(0, bucket.reshape(-1), ds.reshape(-1))
                grads["dbias"][1][:, h].index_add_(0, bucket.reshape(-1), one.reshape(-1))
        qa, ka = qa + nq, ka + room
    res = {"out": (out, out_e), "lse": (lse, lse_e)}
    if dout is not None:
        res.update({n: tuple(x) for n, x in grads.items()})
    return res


def assert_bounded(got, want, error, what=""):
    """|got - want| <= error and half a step of got's type."""
    g = got.detach().cpu().double()
    tol = error + half_step(got.dtype) * (want.abs() + error) + 1e-30
    bad = ~((g - want).abs() <= tol) & ~(g.isnan() & want.isnan()) & ~(g == want)
    if bool(bad.any()):
        k = int(bad.flatten().nonzero()[0])
        worst = float(((g - want).abs() / tol).nan_to_num(np.inf).max())
        raise AssertionError(f"{what}: {int(bad.sum())} of {bad.numel()} beyond their bound (worst {worst:.2f} times), first at "
                             f"{np.unravel_index(k, tuple(want.shape))}: {g.flatten()[k].item()} against "
                             f"{want.flatten()[k].item()}, bound {tol.flatten()[k].item()}")

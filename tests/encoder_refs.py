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

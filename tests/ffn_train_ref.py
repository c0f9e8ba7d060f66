"""Float64 references of the operators that train a gated FFN, from their formulas, and how
far a result computed in 32 bits and rounded once may be from them.

Every bound is a sum of what each step may lose: a rounding to a type is off by at most
half a step, `half(t)` relative to the value; a sum of n products in fp32, in any order,
by at most n 2^-24 times the sum of the products' magnitudes."""
from __future__ import annotations

import math

import torch

U = 2.0 ** -24  # half a step of fp32


def half(dtype) -> float:
    return torch.finfo(dtype).eps / 2


def d(t):
    return None if t is None else t.double()


def act(name, g):
    """(act, act') of the gate, in float64."""
    if name == "none":
        return g, torch.ones_like(g)
    if name == "silu":
        s = torch.sigmoid(g)
        return g * s, s + g * s * torch.sigmoid(-g)
    p = torch.special.ndtr(g)
    return g * p, p + g * torch.exp(-g * g / 2) / math.sqrt(2 * math.pi)


def act_error(name, g, exact):
    """Of act(g) relative to itself, in fp32 arithmetic.
    GELU: (13 + a + 2 a^2) 2^-24 with the fit of the tail, and in a bf16 layer (exact False)
    5.7e-7 e^(1.5 a) more, but never more than 2.8e-3 of it.
    SiLU: e^-g from 2^(-g log2 e): the argument's two roundings move it by 2 |g| 2^-24 of
    itself, the power, the sum, the reciprocal and the product by some 8 2^-24 together."""
    a = g.abs()
    if name == "none":
        return torch.zeros_like(g)
    if name == "silu":
        return (8 + 2 * a) * U
    e = (13 + a + 2 * a * a) * U
    return e if exact else e + torch.clamp(5.7e-7 * torch.exp(torch.clamp(1.5 * a, max=50.0)), max=2.8e-3)


def grad_error(name, g):
    """Of act'(g), absolute: its terms are at most 1.2, a few roundings each and the error of
    act's parts (fp32 throughout)."""
    return (20 + 4 * g.abs().clamp(max=30.0)) * U


def gated(x, W, bias, name):
    """(h, pre, bound of h, bound of pre) of a gated layer over rows x [R, K]."""
    x64, W64 = x.double(), W.double()
    F, K = W.shape[0] // 2, W.shape[1]
    pre, size = x64 @ W64.t().contiguous(), x64.abs() @ W64.abs().t().contiguous()
    if bias is not None:
        pre, size = pre + bias.double(), size + bias.double().abs()
    off = (K + 2) * U * size
    g, u = pre[:, :F], pre[:, F:]
    a, da = act(name, g)
    h = a * u
    # the act's slope is at most 1.2 anywhere within the error of g
    hoff = 1.2 * off[:, :F] * (u.abs() + off[:, F:]) + a.abs() * off[:, F:]
    hoff = hoff + (act_error(name, g, x.dtype == torch.float32) + 2 * U) * h.abs()
    r = half(x.dtype)
    return h, pre, hoff * (1 + r) + r * h.abs() + 1e-37, off * (1 + r) + r * pre.abs() + 1e-37


def products(dy, x, W, off=None):
    """(dx, dW, dbias) of a layer from dy [R, N] in float64, and their bounds; off: how far
    each operand dy may itself be (the gated layer's), and that before its rounding."""
    R, N = dy.shape
    K = x.shape[1]
    x64, W64 = x.double(), W.double()
    r = half(x.dtype)
    dx, dW, db = dy @ W64, dy.t().contiguous() @ x64, dy.sum(0)
    o, raw = (torch.zeros_like(dy),) * 2 if off is None else off
    bx = (o @ W64.abs() + (N + 1) * U * ((dy.abs() + o) @ W64.abs())) * (1 + r) + r * dx.abs() + 1e-37
    bW = (o.t().contiguous() @ x64.abs() + (R + 1) * U * ((dy.abs() + o).t().contiguous() @ x64.abs())) * (1 + r)
    return (dx, dW, db), (bx, bW + r * dW.abs() + 1e-37, raw.sum(0) + (R + 1) * U * (dy.abs() + raw).sum(0) + 1e-37)


def gated_backward(dh, x, W, pre, name):
    F = W.shape[0] // 2
    dh64, g, u = dh.double(), pre[:, :F].double(), pre[:, F:].double()
    a, da = act(name, g)
    dg, du = dh64 * u * da, dh64 * a
    dpre = torch.cat([dg, du], 1)
    raw = torch.cat([(dh64 * u).abs() * grad_error(name, g) + 3 * U * dg.abs(),
                     du.abs() * (act_error(name, g, True) + 2 * U)], 1) + 1e-38
    r = half(x.dtype) if x.dtype != torch.float32 else 0.0
    return products(dpre, x, W, (raw + r * (dpre.abs() + raw), raw))


def norm_stats(t, rms, eps):
    mean = torch.zeros(t.shape[0], dtype=torch.float64, device=t.device) if rms else t.mean(1)
    return mean, ((t - mean[:, None]).square().mean(1) + eps).rsqrt()


def residual(x, b, post, scale, gate, norm, rms, eps):
    """s, y and the four statistics, in float64, of rows [R, C]; gate [R] or None."""
    n, mb, rb, y, ms, rs = b.double(), None, None, None, None, None
    shift = lambda w: 0.0 if w[1] is None else w[1].double()  # noqa: E731
    size = lambda w: 1.0 if w[0] is None else w[0].double()  # noqa: E731
    if post is not None:
        mb, rb = norm_stats(n, rms, eps)
        n = (n - mb[:, None]) * rb[:, None] * size(post) + shift(post)
    f = torch.ones_like(n) if scale is None else scale.double().expand_as(n)
    f = f if gate is None else f * gate.double()[:, None]
    s = x.double() + f * n
    if norm is not None:
        ms, rs = norm_stats(s, rms, eps)
        y = (s - ms[:, None]) * rs[:, None] * size(norm) + shift(norm)
    return s, y, mb, rb, ms, rs


def residual_bounds(x, b, post, scale, gate, norm, rms, eps, want):
    """How far residual's results, `want`, may be off in fp32, the rounding to x's type in."""
    s, y, mb, rb, ms, rs = want
    C = x.shape[1]
    r = half(x.dtype)

    def of(t, off, mean, rstd):
        """Bounds of mean, rstd and (t - mean) rstd for values t that are themselves off."""
        m = torch.zeros_like(mean) if rms else off.mean(1) + (C + 3) * U * t.abs().mean(1)
        dev = off + m[:, None] + 2 * U * (t.abs() + mean.abs()[:, None])
        a = (t - mean[:, None]).abs()
        var = a.square().mean(1)
        v = (2 * a * dev + dev * dev).mean(1) + (C + 3) * U * var + 2 * U * (var + eps)
        q = v * rstd * rstd / 2
        q = torch.where(q < 0.2, q * 1.5 + 3 * U, torch.full_like(q, math.inf))
        return m + 1e-38, q * rstd, dev * rstd[:, None] * (1 + q)[:, None] + a * (rstd * (q + 2 * U))[:, None]

    n, off = b.double(), torch.zeros_like(want[0])
    out = [None] * 6
    size = lambda w: torch.ones(C, dtype=torch.float64, device=b.device) if w[0] is None else w[0].double().abs()  # noqa: E731
    shift = lambda w: 0.0 if w[1] is None else w[1].double()  # noqa: E731
    if post is not None:
        out[2], out[3], z = of(n, off, mb, rb)
        zn = (n - mb[:, None]) * rb[:, None] * (1.0 if post[0] is None else post[0].double())
        n = zn + shift(post)
        off = z * size(post) + U * zn.abs() + U * n.abs()
    f = torch.ones_like(n) if scale is None else scale.double().abs().expand_as(n)
    f = f if gate is None else f * gate.double().abs()[:, None]
    off = f * off * (1 + 2 * U) + 2 * U * f * n.abs() + U * s.abs()
    out[0] = off * (1 + r) + r * s.abs() + 1e-37
    if norm is not None:
        out[4], out[5], z = of(s, off, ms, rs)
        out[1] = (z * size(norm) + U * (y - shift(norm)).abs() + U * y.abs()) * (1 + r) + r * y.abs() + 1e-37
    return out


def residual_backward(ds, dy, b, s, stats, post, scale, gate, norm, rms):
    """{name: (gradient, bound)} in float64; dgate row by row.  A bound is 2^-24 times the sum
    of the magnitudes of what is added, times how many of them there are; (t - mean) rstd
    counts as (|t| + |mean|) rstd, which covers its subtraction."""
    mb, rb, ms, rs = (d(t) for t in stats)
    R, C = b.shape
    like = dict(dtype=torch.float64, device=b.device)
    one = lambda w: torch.ones(C, **like) if w[0] is None else w[0].double()  # noqa: E731
    b64, r = b.double(), half(b.dtype)
    avg = lambda t: t.mean(1, keepdim=True)  # noqa: E731

    def back(h, hs, t, mean, rstd):
        """The norm's gradient of h, its size from h's size, the normalised t and its size."""
        mean = torch.zeros(R, 1, **like) if rms else mean[:, None]
        z, zs = (t - mean) * rstd[:, None], (t.abs() + mean.abs()) * rstd[:, None]
        k = h - z * avg(h * z)
        m = hs + zs * avg(hs * zs)
        if not rms:
            k, m = k - avg(h), m + avg(hs)
        return k * rstd[:, None], m * rstd[:, None], z, zs

    dv = torch.zeros(R, C, **like) if ds is None else ds.double()
    size, out = dv.abs(), {}
    if dy is not None:
        h = dy.double() * one(norm)
        k, m, z, zs = back(h, h.abs(), s.double(), ms, rs)
        dv, size = dv + k, size + m
        dy64 = dy.double()
        out["dnorm"] = (dy64 * z).sum(0), (R + 5) * U * (dy64.abs() * zs).sum(0)
        out["dnorm_bias"] = dy64.sum(0), (R + 1) * U * dy64.abs().sum(0)
    n1 = C + 12  # additions and roundings in each value of dv, and again in each average of k
    out["dx"] = dv, n1 * U * size + r * dv.abs()
    f = torch.ones(R, C, **like) if scale is None else scale.double().expand(R, C)
    g = torch.ones(R, 1, **like) if gate is None else gate.double()[:, None]
    dn, dns, n, ns = dv * f * g, size * (f * g).abs(), b64, b64.abs()
    db, dbs = dn, dns
    if post is not None:
        db, dbs, z, zs = back(dn * one(post), dns * one(post).abs(), b64, mb, rb)
        shift = torch.zeros(C, **like) if post[1] is None else post[1].double()
        n, ns = z * one(post) + shift, zs * one(post).abs() + shift.abs()
        out["dpost"] = (dn * z).sum(0), (R + n1 + 5) * U * (dns * zs).sum(0)
        out["dpost_bias"] = dn.sum(0), (R + n1 + 5) * U * dns.sum(0)
    out["db"] = db, 2 * n1 * U * dbs + r * db.abs()
    out["dscale"] = (dv * g * n).sum(0), (R + n1 + 8) * U * (size * g.abs() * ns).sum(0)
    out["dgate"] = (dv * f * n).sum(1), (C + n1 + 8) * U * (size * f.abs() * ns).sum(1)
    return {k: (v, e * 1.01 + 1e-37) for k, (v, e) in out.items()}

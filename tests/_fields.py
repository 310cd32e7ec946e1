"""Plain 64-bit forms of group norm with an activation, and the error that the
kernels' arithmetic allows, element by element (as _layers: a result's own rounding
comes on top).  u = 2^-24 is an fp32 rounding."""
import torch

from _layers import ACTS, DT, EPS32, act64, sum_error   # noqa: F401

EPS = 1e-5


def field(gen, shape, dtype, scale=1.0, shift=0.0, pad=0, spad=0, offset=0):
    """[.., S, P, C] on the device, points C + pad elements apart, samples spad more
    than their points, the first element `offset` into its buffer; NaN between."""
    *lead, S, P, C = shape
    G = lead[0] if lead else 1
    ld = C + pad
    ss = max(P, 1) * ld + spad
    gs = max(S, 1) * ss + 3 * bool(spad)
    buf = torch.full((G * gs + offset + 8,), float("nan"), dtype=torch.float32).to(DT[dtype]).cuda()
    t = buf.as_strided((G, S, P, C), (gs, ss, ld, 1), offset)
    v = torch.randn((G, S, P, C), generator=gen, dtype=torch.float32) * scale + shift
    t.copy_(v.to(DT[dtype]))
    return t if lead else t[0]


def _wide(t, n):
    """[.., C] or [.., S, P, C] as [.., n, c]"""
    return t.unflatten(-1, (n, t.shape[-1] // n))


def forward64(x, n, gamma, beta, act):
    """(y, mean, rstd, error of y) in 64 bits, on the host; gamma and beta [.., C].

    The mean is rounded (u |mean|), then its difference, rstd, rstd gamma, their
    product and the sum with beta; an activation's slope is at most 1.13."""
    xs = _wide(x.double().cpu(), n)                      # [.., S, P, n, c]
    ga, be = (_wide(t.double().cpu(), n)[..., None, None, :, :] for t in (gamma, beta))
    mean = xs.mean((-3, -1), keepdim=True)
    var = (xs - mean).square().mean((-3, -1), keepdim=True)
    rstd = (var + EPS) ** -0.5
    xh = (xs - mean) * rstd
    a = xh * ga + be
    err = EPS32 * ((mean * rstd * ga).abs() + 4 * (xh * ga).abs() + a.abs())
    err = 1.13 * err + act_error(a, act, x.dtype)
    stats = (*x.shape[:-2], n)
    return act64(a, act)[0].reshape(x.shape), mean.reshape(stats), rstd.reshape(stats), err.reshape(x.shape)


def act_error(a, act, dtype):
    """of an activation or its slope: 2e-6 in fp32, 1e-8 in fp64"""
    if act == "none":
        return torch.zeros_like(a)
    return (1e-8 if dtype == torch.float32 else 2e-6) * (1 + a.abs())


def backward64(dy, x, mean, rstd, gamma, beta, act, add=None):
    """((dx, its error), (dgamma, error), (dbeta, error)) in 64 bits, on the host, at
    the statistics given."""
    n = mean.shape[-1]
    xs, d = _wide(x.double().cpu(), n), _wide(dy.double().cpu(), n)
    ga, be = (_wide(t.double().cpu(), n)[..., None, None, :, :] for t in (gamma, beta))
    mu, rs = (t.double().cpu()[..., None, :, None] for t in (mean, rstd))
    N = xs.shape[-3] * xs.shape[-1]
    xh = (xs - mu) * rs
    e_xh = 2 * EPS32 * xh.abs()
    a = xh * ga + be
    e_a = ga.abs() * e_xh + EPS32 * ((xh * ga).abs() + a.abs())
    slope = act64(a, act)[1]
    # second derivatives are at most 1; relu's slope jumps where a may have either sign
    e_slope = act_error(a, act, x.dtype) + (e_a if act != "none" else 0)
    if act == "relu":
        e_slope = e_slope + (a.abs() <= e_a)
    da = d * slope
    e_da = d.abs() * e_slope + EPS32 * da.abs()
    h = da * ga
    e_h = e_da * ga.abs() + EPS32 * h.abs()

    def mean_of(v, e):
        over = (-3, -1)
        m = v.mean(over, keepdim=True)
        rss = v.square().sum(over, keepdim=True).sqrt()
        return m, e.mean(over, keepdim=True) + sum_error(N, 1.0) * rss / N + EPS32 * m.abs()

    m1, e1 = mean_of(h, e_h)
    m2, e2 = mean_of(h * xh, e_h * xh.abs() + h.abs() * e_xh + EPS32 * (h * xh).abs())
    dx = rs * (h - m1 - xh * m2)
    e = rs * (e_h + e1 + xh.abs() * e2 + m2.abs() * e_xh + 4 * EPS32 * (h.abs() + m1.abs() + (xh * m2).abs()))
    dx, e = dx.reshape(x.shape), e.reshape(x.shape)
    if add is not None:
        dx = dx + add.double().cpu()
        e = e + EPS32 * dx.abs()

    def cols(v, e):
        over = (-4, -3)
        rss = v.square().sum(over).sqrt()
        rows = v.shape[-4] * v.shape[-3]
        t = v.sum(over)
        err = e.sum(over) + sum_error(rows, 1.0) * rss
        shape = (*v.shape[:-4], x.shape[-1])
        return t.reshape(shape), err.reshape(shape)

    return (dx, e), cols(da * xh, e_da * xh.abs() + da.abs() * e_xh + EPS32 * (da * xh).abs()), cols(da, e_da)

"""Plain 64-bit forms of the linear layer and of layer norm, and the error that
the kernels' arithmetic allows, element by element.

A result is rounded once to its type (unit u: half a unit in the last place,
relative).  Before that, a sum of n products in fp32 is off by at most the
roundings of its partial sums; those are independent and a partial sum stays
within a few times rss = sqrt(sum of squared products), so 32 sqrt(n) 2^-24 rss
is many standard deviations.  The activations are evaluated to 2e-6 (relative to
1 + |a|) in fp32, and their slopes are at most 1.13."""
import math

import torch

DT = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}
UNIT = {"fp32": 2.0 ** -24, "bf16": 2.0 ** -8, "fp16": 2.0 ** -11}   # 24, 8 and 11 significand bits
TINY = {"fp32": 2.0 ** -126, "bf16": 2.0 ** -126, "fp16": 2.0 ** -25}   # spacing below the normal range
EPS32 = 2.0 ** -24
ACTS = ("none", "tanh", "relu", "gelu", "silu")


def act64(a, act):
    """(act(a), act'(a))"""
    if act == "tanh":
        return a.tanh(), a.cosh() ** -2
    if act == "relu":
        return a.clamp(min=0), (a > 0).double()
    if act == "gelu":
        cdf = torch.special.ndtr(a)
        return a * cdf, cdf + a * torch.exp(-a * a / 2) / math.sqrt(2 * math.pi)
    if act == "silu":
        s = torch.sigmoid(a)
        return a * s, s * (1 + a * (1 - s))
    return a, torch.ones_like(a)


def matrix(gen, G, rows, cols, dtype, scale=1.0, shift=0.0, ld=None, offset=0):
    """[G, rows, cols] ([rows, cols] for G = None) on the device, rows `ld`
    elements apart, the first one `offset` elements into its buffer; NaN between
    the rows."""
    ld = ld or cols
    g = G or 1
    buf = torch.full((g * max(rows, 1) * ld + offset + 8,), float("nan"), dtype=torch.float32)
    v = torch.randn((g, rows, cols), generator=gen, dtype=torch.float32) * scale + shift
    t = buf.to(DT[dtype]).cuda()
    m = t.as_strided((g, rows, cols), (max(rows, 1) * ld, ld, 1), offset)
    m.copy_(v.to(DT[dtype]))
    return m if G else m[0]


def vector(gen, G, cols, scale=1.0, shift=0.0):
    v = (torch.randn((G or 1, cols), generator=gen, dtype=torch.float32) * scale + shift).cuda()
    return v if G else v[0]


def mm64(a, b):
    """(a b^T, root of the sum of squared products) in 64 bits, on the host"""
    a, b = a.double().cpu(), b.double().cpu()
    return a @ b.transpose(-1, -2), ((a * a) @ (b * b).transpose(-1, -2)).sqrt()


def sum_error(n, rss):
    return 32 * math.sqrt(n + 16) * EPS32 * rss


def check(got, want, error, dtype, what):
    """|got - want| within `error` before the rounding to dtype"""
    got = got.double().cpu()
    tol = error + UNIT[dtype] * (want.abs() + error) + TINY[dtype]
    bad = ~((got - want).abs() <= tol)
    assert got.shape == want.shape
    if bad.any():
        i = int(bad.flatten().nonzero()[0])
        raise AssertionError(f"{what}: {int(bad.sum())} of {bad.numel()} elements off, the first at {i}: "
                             f"{got.flatten()[i]} for {want.flatten()[i]}, tolerance {tol.flatten()[i]}")

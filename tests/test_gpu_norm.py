"""Layer norm and the reverse pass of an activation against their formulas in
64 bits: row lengths around every variant, single rows to many, odd strides,
groups, constant rows, values that are not finite."""
import math

import pytest
import torch

from paper_1910_13444_amd import pigan
from _layers import ACTS, EPS32, act64, check, matrix, sum_error, vector

pytestmark = pytest.mark.gpu

F32 = dict(device="cuda", dtype=torch.float32)

EPS = 1e-5
# row lengths: one column, tails of pieces, each number of threads per row (16-bit
# and fp32 rows have pieces of 8 and 4), and rows that no block holds in registers
COLS = [1, 3, 8, 33, 64, 129, 256, 257, 500, 512, 1001, 1024, 1025, 2048, 4097, 8191, 16384, 16391, 40000]
ROWS = [1, 2, 7, 130, 1000]


def _seed(*a):
    g = torch.Generator()
    g.manual_seed(hash(a) % (1 << 31))
    return g


def _depth(N):
    """Additions that one of a row's values takes part in: a thread's pieces,
    the lanes and waves of the row; rows beyond 1024 threads' registers turn
    N / 1024 times."""
    return 64 + N / 1024


def _forward(gen, G, M, N, dtype, shift=0.5, ld=lambda c: c, offset=0, affine=True):
    x = matrix(gen, G, M, N, dtype, shift=shift, ld=ld(N), offset=offset)
    out = matrix(gen, G, M, N, dtype, ld=ld(N), offset=offset)
    ga, be = (vector(gen, G, N, 0.2, 1.0), vector(gen, G, N, 0.2)) if affine else (None, None)
    y, mean, rstd = pigan.layer_norm(x, ga, be, eps=EPS, out=out)
    torch.cuda.synchronize()
    x64 = x.double().cpu()
    m = x64.mean(-1, keepdim=True)
    var = (x64 - m).square().mean(-1, keepdim=True)
    r = (var + EPS) ** -0.5
    size = x64.abs().amax(-1, keepdim=True)
    e_mean = _depth(N) * EPS32 * size
    check(mean, m.squeeze(-1), e_mean.squeeze(-1), "fp32", "mean")
    # var is off by the roundings of its sum and the square of the mean's error
    e_var = (_depth(N) + 8) * EPS32 * var + 4 * EPS32 * size * var.sqrt() + e_mean ** 2
    e_rel = 0.5 * e_var / (var + EPS) + 4 * EPS32
    check(rstd, r.squeeze(-1), (r * e_rel).squeeze(-1), "fp32", "rstd")
    g64 = ga.double().cpu().unsqueeze(-2) if affine else 1.0
    b64 = be.double().cpu().unsqueeze(-2) if affine else 0.0
    xh = (x64 - m) * r
    want = xh * g64 + b64
    err = (xh.abs() * (e_rel + 4 * EPS32) + (e_mean + EPS32 * size) * r) * (g64.abs() if affine else 1.0)
    check(y, want, err + 2 * EPS32 * want.abs(), dtype, "y")
    return x, mean, rstd, ga


@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("N", COLS)
def test_forward_columns(N, dtype):
    print(f"norm forward {N} {dtype}", flush=True)
    _forward(_seed(N), None, 11, N, dtype)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("M", ROWS)
@pytest.mark.parametrize("N", [24, 300, 4000])
def test_forward_rows(M, N, dtype):
    _forward(_seed(M, N), None, M, N, dtype, affine=M != 7)


@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("pad,offset", [(8, 0), (3, 1), (0, 5)])
@pytest.mark.parametrize("N", [100, 1000, 20000])
def test_strides_and_groups(dtype, pad, offset, N):
    _forward(_seed(N), 3, 5, N, dtype, ld=lambda c: c + pad, offset=offset)
    _backward(_seed(N), 3, 5, N, dtype, True, ld=lambda c: c + pad, offset=offset)


def test_forward_does_not_cancel():
    """A row far from zero keeps its variance."""
    for N in (40, 700, 20000):
        _forward(_seed(N), None, 6, N, "fp32", shift=1000.0)


def test_constant_rows_and_in_place():
    for N in (1, 65, 2000, 40000):
        x = torch.full((4, N), 3.0, **F32)
        y, mean, rstd = pigan.layer_norm(x, eps=EPS)
        assert not y.any() and torch.equal(mean, torch.full((4,), 3.0, **F32))
        torch.testing.assert_close(rstd, torch.full((4,), EPS ** -0.5, **F32), rtol=1e-6, atol=0)
        x = matrix(_seed(N), None, 4, N, "fp32")
        y, _, _ = pigan.layer_norm(x, eps=EPS)
        pigan.layer_norm(x, eps=EPS, out=x)
        assert torch.equal(x, y)


def _backward(gen, G, M, N, dtype, add, ld=lambda c: c, offset=0, affine=True):
    x = matrix(gen, G, M, N, dtype, shift=0.5, ld=ld(N), offset=offset)
    dy = matrix(gen, G, M, N, dtype, scale=0.3, ld=ld(N), offset=offset)
    r = matrix(gen, G, M, N, dtype, ld=ld(N), offset=offset) if add else None
    out = matrix(gen, G, M, N, dtype, ld=ld(N), offset=offset)
    ga = vector(gen, G, N, 0.2, 1.0) if affine else None
    x64, d64 = x.double().cpu(), dy.double().cpu()
    m = x64.mean(-1)
    s = ((x64 - m.unsqueeze(-1)).square().mean(-1) + EPS) ** -0.5
    mean, rstd = m.float().cuda(), s.float().cuda()
    dx, dgamma, dbeta = pigan.layer_norm_backward(dy, x, mean, rstd, ga, add=r, dx=out)
    torch.cuda.synchronize()
    m, s = mean.double().cpu().unsqueeze(-1), rstd.double().cpu().unsqueeze(-1)
    xh = (x64 - m) * s
    h = d64 * (ga.double().cpu().unsqueeze(-2) if affine else 1.0)
    h1, h2 = h.mean(-1, keepdim=True), (h * xh).mean(-1, keepdim=True)
    want = s * (h - h1 - xh * h2)
    e1 = (_depth(N) + 8) * EPS32
    err = s * (4 * EPS32 * h.abs() + e1 * h.abs().mean(-1, keepdim=True) +
               xh.abs() * e1 * (h * xh).abs().mean(-1, keepdim=True) + 8 * EPS32 * (h1.abs() + (xh * h2).abs()))
    if add:
        want = want + r.double().cpu()
        err = err + EPS32 * want.abs()
    check(dx, want, err, dtype, "dx")
    t = d64 * xh
    check(dgamma, t.sum(-2), sum_error(M, (t * t).sum(-2).sqrt()) + 4 * EPS32 * t.abs().sum(-2), "fp32", "dgamma")
    check(dbeta, d64.sum(-2), sum_error(M, (d64 * d64).sum(-2).sqrt()), "fp32", "dbeta")
    return dy, x, mean, rstd, ga, r, dx, dgamma, dbeta


@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("N", COLS)
def test_backward_columns(N, dtype):
    print(f"norm backward {N} {dtype}", flush=True)
    _backward(_seed(N), None, 11, N, dtype, N % 2 == 0)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("M", ROWS + [6000])
@pytest.mark.parametrize("N", [24, 300, 1500])
def test_backward_rows(M, N, dtype):
    _backward(_seed(M, N), None, M, N, dtype, True, affine=M != 7)


@pytest.mark.parametrize("N", [40, 900, 3000, 20000])
def test_backward_parts_and_in_place(N):
    dy, x, mean, rstd, ga, r, dx, dg, db = _backward(_seed(N), None, 300, N, "bf16", True)
    a = pigan.layer_norm_backward(dy, x, mean, rstd, ga, add=r, need_params=False)
    b = pigan.layer_norm_backward(dy, x, mean, rstd, ga, need_dx=False)
    assert torch.equal(a[0], dx) and torch.equal(b[1], dg) and torch.equal(b[2], db) and b[0] is None and a[1] is None
    p, q = dy.clone(), r.clone()
    c = pigan.layer_norm_backward(p, x, mean, rstd, ga, add=r, dx=p)
    d = pigan.layer_norm_backward(dy, x, mean, rstd, ga, add=q, dx=q)
    for o in (c, d):
        assert torch.equal(o[0], dx) and torch.equal(o[1], dg) and torch.equal(o[2], db)


def test_gradients_are_differences():
    gen = _seed(3)
    M, N, h = 9, 70, 2.0 ** -6
    x0, ga0, be0 = matrix(gen, None, M, N, "fp32"), vector(gen, None, N, 0.2, 1.0), vector(gen, None, N)
    c = matrix(gen, None, M, N, "fp32")

    def f(x, ga, be):
        return float((pigan.layer_norm(x, ga, be)[0].double() * c.double()).sum())

    _, mean, rstd = pigan.layer_norm(x0, ga0, be0)
    dx, dg, db = pigan.layer_norm_backward(c, x0, mean, rstd, ga0)
    scale = float((dx.double() ** 2).sum() + (dg.double() ** 2).sum() + (db.double() ** 2).sum()) ** 0.5
    for k in range(6):
        vx, vg, vb = matrix(gen, None, M, N, "fp32"), vector(gen, None, N), vector(gen, None, N)
        num = (f(x0 + h * vx, ga0 + h * vg, be0 + h * vb) - f(x0 - h * vx, ga0 - h * vg, be0 - h * vb)) / (2 * h)
        ana = float((dx.double() * vx).sum() + (dg.double() * vg).sum() + (db.double() * vb).sum())
        assert abs(num - ana) <= 0.02 * scale, (k, num, ana, scale)


def test_no_rows_and_nonfinite():
    for dtype in (torch.float32, torch.bfloat16):
        x = torch.empty((0, 50), dtype=dtype, device="cuda")
        y, mean, rstd = pigan.layer_norm(x)
        assert y.shape == (0, 50) and mean.shape == (0,)
        dg, db = torch.full((50,), 7.0, **F32), torch.full((50,), 7.0, **F32)
        pigan.layer_norm_backward(x, x, mean, rstd, dgamma=dg, dbeta=db)
        assert not dg.any() and not db.any()
        for N in (20, 300, 5000, 20000):
            x = torch.randn((40, N), device="cuda").to(dtype)
            clean = pigan.layer_norm(x)
            x[39, N - 1] = math.nan
            y, mean, rstd = pigan.layer_norm(x)
            assert torch.equal(y[:39], clean[0][:39]) and torch.isnan(y[39]).all() and torch.isnan(mean[39])


@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("act", ACTS[1:])
@pytest.mark.parametrize("G,M,N,pad,offset", [(None, 1, 1, 0, 0), (None, 128, 32, 0, 0), (None, 33, 77, 3, 1),
                                              (4, 19, 200, 8, 0), (None, 3000, 1001, 0, 0), (None, 1, 100000, 0, 0)])
def test_act_backward(dtype, act, G, M, N, pad, offset):
    gen = _seed(M, N)
    dy = matrix(gen, G, M, N, dtype, ld=N + pad, offset=offset)
    pre = matrix(gen, G, M, N, dtype, scale=3.0, ld=N + pad, offset=offset)
    g = pigan.act_backward(dy, pre, act)
    torch.cuda.synchronize()
    s = act64(pre.double().cpu(), act)[1]
    d = dy.double().cpu()
    check(g, d * s, d.abs() * 4e-6, dtype, "g")
    assert torch.equal(pigan.act_backward(dy, pre, act, out=dy), g)


def test_activation_range():
    """Values and slopes far out and around zero: relative to 1 + |a|, finite
    wherever the formula is."""
    far = torch.tensor([0.0, -0.0, 1e-30, -1e-30, 90.0, -90.0, 1e4, -1e4, 1e30, -1e30])
    a = torch.cat([torch.linspace(-30, 30, 6001), far]).to(**F32)
    one = torch.ones((1, 1), **F32)
    for act in ACTS[1:]:
        v, s = act64(a.double().cpu(), act)
        y = pigan.linear(a[:, None].contiguous(), one, act=act)[:, 0]
        g = pigan.act_backward(torch.ones_like(a)[None], a[None], act)[0]
        torch.cuda.synchronize()
        check(y, v, 2e-6 * (1 + a.double().cpu().abs().clamp(max=1)) * v.abs().clamp(min=1), "fp32", act)
        check(g, s, torch.full_like(s, 4e-6), "fp32", act + " slope")

"""fp32 products of the linear layer: every significand bit of the operands, every
pair of planes in every tile and split, infinities as in the formula."""
import math

import pytest
import torch

from paper_1910_13444_amd import pigan
from _layers import DT, EPS32, check, matrix, mm64, sum_error
from test_gpu_linear import _seed
from test_gpu_linear_tiles import BACKWARD32, FORWARD32

pytestmark = pytest.mark.gpu

F32 = dict(device="cuda", dtype=torch.float32)


def _planes(x):
    """x as three bf16 values that add up to it, in 64 bits"""
    x0 = x.bfloat16().float()
    x1 = (x - x0).bfloat16().float()
    return x0.double(), x1.double(), (x - x0 - x1).double()


def _values(gen, n):
    """significands with every bit in use, and those whose lower bits are largest"""
    hard = [1 + 2.0 ** -7 - 2.0 ** -23, 1 + 2.0 ** -8, 1 + 2.0 ** -8 - 2.0 ** -23, 2 - 2.0 ** -23, 1 + 2.0 ** -8 + 2.0 ** -17,
            1 + 2.0 ** -8 - 2.0 ** -17 + 2.0 ** -23, 1.0, 1.5]
    v = torch.cat([torch.tensor(hard, dtype=torch.float32), torch.rand(n - len(hard), generator=gen, dtype=torch.float32) + 1])
    return v * (torch.randint(0, 2, (n,), generator=gen) * 2 - 1)


def test_single_products():
    """Contractions of one element: a product loses at most 2^-24 of itself to the
    pairs of planes that are left out, and two roundings of the sum of the six, each
    at most a unit (2^-23) should the matrix core cut."""
    gen = _seed(1)
    a, b = _values(gen, 1011).cuda(), _values(gen, 777).cuda()
    want = a.double()[:, None] * b.double()[None, :]
    bound = (1 + 2 * 2) * EPS32 * want.abs()
    dw = pigan.linear_backward(a[None, :], b[None, :], torch.zeros((1011, 777), **F32), need_dx=False)[1]
    assert ((dw.double() - want).abs() <= bound).all()
    dx = pigan.linear_backward(a[:, None], torch.zeros((1011, 777), **F32), b[None, :], need_dw=False)[0]
    assert ((dx.double() - want).abs() <= bound).all()
    # rows enough for the tiles
    a = _values(gen, 150001).cuda()
    y = pigan.linear(a[:, None], b[:, None])
    want = a.double()[:, None] * b.double()[None, :]
    assert ((y.double() - want).abs() <= (1 + 2 * 2) * EPS32 * want.abs()).all()


def test_largest_values():
    """A value whose nearest bf16 is infinite."""
    big = torch.tensor([3.4028234663852886e38, -3.4028234663852886e38, 3.39e38], **F32)
    dw = pigan.linear_backward(big[None, :], torch.full((1, 500), 0.375, **F32), torch.zeros((3, 500), **F32), need_dx=False)[1]
    want = big.double()[:, None] * 0.375
    assert ((dw.double() - want).abs() <= 5 * EPS32 * want.abs()).all()


def _rms(t):
    return t.square().mean().sqrt().item()


def _judge(got, a, b, what):
    """got = a b^T for unit normals.  A partial sum of k products is sqrt(k) in the
    root mean square, and rounding it to nearest is off by 0.42 * 2^-24 of that: n
    additions one by one by 0.3 n units of 2^-24, cut sums by half as much again at
    sqrt(n) (their errors have both signs as the sums have); the final rounding and
    the pairs left out by less than sqrt(n) together.  The pair (1, 1) left out as
    well would show."""
    n = a.shape[-1]
    want = a.double() @ b.double().transpose(-1, -2).contiguous()
    tol = (0.45 * n + math.sqrt(n)) * EPS32
    err = _rms(got.double() - want)
    assert err <= tol, f"{what}: {err / EPS32} units for at most {tol / EPS32}"
    if n >= 100 and n <= 2000:
        (_, a1, _), (_, b1, _) = _planes(a), _planes(b)
        assert _rms(a1 @ b1.transpose(-1, -2).contiguous()) > tol, f"{what}: a missing pair would pass"


@pytest.mark.parametrize("size", FORWARD32)
def test_every_pair_forward(size):
    G, M, K, N = size
    gen = _seed(*size)
    x, w = matrix(gen, G, M, K, "fp32"), matrix(gen, G, N, K, "fp32")
    _judge(pigan.linear(x, w), x, w, "y")


@pytest.mark.parametrize("size", BACKWARD32)
def test_every_pair_backward(size):
    G, M, K, N = size
    gen = _seed(*size)
    g, x, w = matrix(gen, G, M, N, "fp32"), matrix(gen, G, M, K, "fp32"), matrix(gen, G, N, K, "fp32")
    dx, dw, _ = pigan.linear_backward(g, x, w)
    _judge(dx, g, w.transpose(-1, -2), "dx")
    _judge(dw, g.transpose(-1, -2), x.transpose(-1, -2), "dw")


def test_fp32_rows_too_wide_for_buffers():
    """Planes whose rows are 2^21 values and more apart."""
    M, K, N = 70, 2 ** 21 + 3, 9
    gen = torch.Generator(device="cuda").manual_seed(9)
    x, w, g = (torch.randn(shape, generator=gen, **F32) for shape in ((M, K), (N, K), (M, N)))
    _judge(pigan.linear(x, w), x, w, "y")
    dx, dw, _ = pigan.linear_backward(g, x, w)
    _judge(dx, g, w.t(), "dx")
    _judge(dw, g.t(), x.t(), "dw")
    # k along rows that wide: a layer of 9 inputs
    dx = pigan.linear_backward(x, g, w.t().contiguous(), need_dw=False)[0]
    _judge(dx, x, w, "dx of a wide cotangent")


def _same(got, a, b, dtype, what):
    """as the formula: the same infinities and NaN, the other elements close"""
    want, _ = mm64(a, b)
    _, rss = mm64(torch.nan_to_num(a.float(), 0, 0, 0), torch.nan_to_num(b.float(), 0, 0, 0))
    got = got.double().cpu()
    assert torch.equal(got.isnan(), want.isnan()), f"{what}: NaN"
    assert torch.equal(got.isinf(), want.isinf()) and torch.equal(got[want.isinf()], want[want.isinf()]), f"{what}: infinities"
    fin = want.isfinite()
    check(got[fin], want[fin], sum_error(a.shape[-1], rss)[fin], dtype, what)


@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("M,K,N", [(12, 200, 140), (600, 200, 140), (64, 200, 140), (2100, 520, 264)])
def test_infinities_follow_the_formula(dtype, M, K, N):
    gen = _seed(29)
    inf = math.inf

    def put(t):
        """infinities of both signs, two in a row, and rows of few significand bits"""
        t[3, 5], t[5, 11], t[7, 20], t[7, 21], t[9, 30], t[9, 31], t[M % 7, 40] = inf, -inf, inf, inf, inf, -inf, math.nan
        return t

    x, w = put(matrix(gen, None, M, K, dtype)), matrix(gen, None, N, K, dtype, scale=0.25)
    w[10:20] = torch.tensor([1.0, 0.5, -1.0, 2.0, -0.5, 0.0, 3.0, -2.0, 1.0, -3.0], dtype=DT[dtype], device="cuda")[:, None]
    w[20, 5], w[21, 5], w[22, 11], w[23, 30], w[24, 50] = inf, -inf, -inf, 0.0, inf
    _same(pigan.linear(x, w), x, w, dtype, "y")
    g = put(matrix(gen, None, M, N, dtype))
    dx, dw, db = pigan.linear_backward(g, x, w)
    _same(dx, g, w.t(), dtype, "dx")
    _same(dw, g.t(), x.t(), "fp32", "dw")
    want = g.double().sum(0)
    assert torch.equal(db.isnan(), want.isnan()) and torch.equal(db[want.isinf()].double(), want[want.isinf()])

"""Group norm at the ends of what it takes: the longest samples, the most channels, the
longest sums.  Fields of gigabytes are compared on the device, in parts, with the formulas
in 64 bits; tolerances as in _fields.py and _layers.py."""
import pytest
import torch

from paper_1910_13444_amd import pigan
from _layers import EPS32, TINY, UNIT, check, sum_error

pytestmark = pytest.mark.gpu

EPS = 1e-5


@pytest.fixture(autouse=True)
def _memory():
    yield
    torch.cuda.empty_cache()


def _parts(n, most=1 << 26):
    for at in range(0, n, most):
        yield slice(at, min(n, at + most))


def _near(got, want, error, dtype):
    """|got - want| within `error` before the rounding to dtype, on the device"""
    return bool(((got.double() - want).abs() <= error + UNIT[dtype] * (want.abs() + error) + TINY[dtype]).all())


@pytest.mark.parametrize("P", [2 ** 31 - 1, 2 ** 31 - 400_000])
def test_the_longest_samples(P):
    """One sample of one channel.  Results go to a buffer whose elements in front of and
    behind them stay as they are: a walk over the points that passed 32 bits would leave them."""
    front, behind, dev = 1 << 20, 1 << 12, "cuda"
    gen = torch.Generator(device=dev).manual_seed(1)
    x, dy = (torch.empty(P, dtype=torch.bfloat16, device=dev) for _ in range(2))
    for k in _parts(P):
        x[k].normal_(0.5, 1.0, generator=gen)
        dy[k].normal_(0.05, 0.1, generator=gen)
    buf = torch.full((front + P + behind,), 7.0, dtype=torch.bfloat16, device=dev)
    out = buf[front:front + P].view(1, P, 1)
    gamma, beta = (torch.full((1,), v, dtype=torch.float32, device=dev) for v in (1.25, -0.5))

    def apart():
        assert bool((buf[:front] == 7).all()) and bool((buf[front + P:] == 7).all())

    _, mean, rstd = pigan.group_norm(x.view(1, P, 1), 1, gamma, beta, out=out)
    torch.cuda.synchronize()
    apart()
    s = sum(x[k].double().sum() for k in _parts(P)) / P
    var = sum((x[k].double() - s).square().sum() for k in _parts(P)) / P
    check(mean.view(()), s.cpu(), 1e-12, "fp32", "mean")
    check(rstd.view(()), (var + EPS).rsqrt().cpu(), 1e-9, "fp32", "rstd")
    m, r, y = mean.double().view(()), rstd.double().view(()), out.view(P)
    for k in _parts(P):
        xh = (x[k].double() - m) * r
        assert _near(y[k], xh * 1.25 - 0.5, EPS32 * (5 * (xh * 1.25).abs() + m.abs() * 2 + 1), "bf16"), k

    dx, dgamma, dbeta = pigan.group_norm_backward(dy.view(1, P, 1), x.view(1, P, 1), mean, rstd, gamma, beta, dx=out)
    torch.cuda.synchronize()
    apart()
    sums = torch.zeros(4, dtype=torch.float64, device=dev)
    for k in _parts(P):
        d, t = dy[k].double(), dy[k].double() * ((x[k].double() - m) * r)
        sums += torch.stack([d.sum(), d.square().sum(), t.sum(), t.square().sum()])
    e_b, e_g = (sum_error(P, 1.0) * sums[i].sqrt() for i in (1, 3))
    e_g = e_g + 4 * EPS32 * (P * sums[3]).sqrt()   # xhat's two roundings of every term and the product's
    check(dbeta.view(()), sums[0].cpu(), e_b.cpu(), "fp32", "dbeta")
    check(dgamma.view(()), sums[2].cpu(), e_g.cpu(), "fp32", "dgamma")
    m1, m2 = 1.25 * sums[0] / P, 1.25 * sums[2] / P
    e_m = 1.25 * (e_b + e_g) / P
    for k in _parts(P):
        xh = (x[k].double() - m) * r
        h = 1.25 * dy[k].double()
        err = r * (e_m * (1 + xh.abs()) + 8 * EPS32 * (h.abs() + m1.abs() + (xh * m2).abs()))
        assert _near(y[k], r * (h - m1 - xh * m2), err, "bf16"), k


def test_more_slabs_than_a_launch_holds():
    """4,198,400 slabs of 64 channels whose 130 points take 1024 threads: more than 2^32.  A
    field of one tile repeated gives the tile's results everywhere, in place (70 GB)."""
    P, W, K = 130, 64 * 4096, 1025
    gen = torch.Generator(device="cuda").manual_seed(2)
    tile = torch.empty((P, W), dtype=torch.bfloat16, device="cuda").normal_(0.5, 1.0, generator=gen)
    gamma, beta = (torch.empty(W, dtype=torch.float32, device="cuda").normal_(v, 0.2, generator=gen) for v in (1.0, 0.0))
    want, mean, rstd = pigan.group_norm(tile.view(1, P, W), W // 64, gamma, beta)
    x = torch.empty((1, P, K * W), dtype=torch.bfloat16, device="cuda")
    wide = x.view(P, K, W)
    wide.copy_(tile[:, None, :].expand(P, K, W))
    y, m, r = pigan.group_norm(x, K * W // 64, gamma.repeat(K), beta.repeat(K), out=x)
    torch.cuda.synchronize()
    assert torch.equal(m.view(K, -1), mean.expand(K, -1)) and torch.equal(r.view(K, -1), rstd.expand(K, -1))
    for p in range(P):
        assert torch.equal(wide[p], want[0, p].expand(K, W)), p


@pytest.mark.parametrize("size", [(1024, 16384, 1, 256, 1), (1024, 172032, 3, 8, 1), (None, 1, 768 * 256 * 4096, 1, 1),
                                  (None, 3072, 4096 * 256, 1, 1)])
def test_long_sums_of_one_sign(size):
    """fp32 gradients of gamma and beta of up to 3e9 equal terms.  The pass sums up to 512
    terms in fp32 (half a unit of the partial sum each) and joins in fp64; 4096 terms of this
    value in a row would be off by 1000 half units."""
    G, S, P, C, n = size
    c = 1.0216064453125
    shape, lead = ((S, P, C), ()) if G is None else ((G, S, P, C), (G,))
    x = torch.full(shape, c, dtype=torch.float32, device="cuda")
    mean, rstd = (torch.full((*lead, S, n), v, dtype=torch.float32, device="cuda") for v in (0.0, 1.0))
    _, dgamma, dbeta = pigan.group_norm_backward(x, x, mean, rstd, need_dx=False)
    torch.cuda.synchronize()
    del x
    for got, term in ((dgamma, c * c), (dbeta, c)):
        want = torch.full((*lead, C), S * P * term, dtype=torch.float64)
        check(got, want, 514 * EPS32 * want, "fp32", "sum")   # and the term's own roundings

"""AdamW at the ends of fp32's range: the step is formed from m and v as they are stored,
an infinite v included.

As in test_gpu_adamw.py the change of a parameter is off by 2^-22 of the quotient's term and
a few fp64 roundings (4e-16 of each term)."""
import math

import pytest
import torch

from paper_1910_13444_amd import pigan
from paper_1910_13444_amd.train import AdamW
from _layers import check

pytestmark = pytest.mark.gpu

LR, B1, B2, EPS, DECAY = 1e-4, 0.5, 0.9, 1e-8, 0.1
MOST = 3.4028234663852886e38


def _states(m, v, g):
    """stored m and v in fp64, infinities and NaN included"""
    return (B1 * m + (1 - B1) * g).float().double(), (B2 * v + (1 - B2) * g * g).float().double()


def _check_step(p, before, m, v, t):
    u = m / (1 - B1 ** t) / ((v / (1 - B2 ** t)).sqrt() + EPS)
    want = before - LR * (u + DECAY * before)
    nan = want.isnan()
    assert torch.equal(p.isnan().cpu(), nan)
    err = 2.0 ** -22 * LR * u.abs() + 4e-16 * (before.abs() + LR * u.abs())
    over = want.abs() > MOST   # none is within err of it
    assert torch.equal(p.cpu()[over], want[over].sign().float() * math.inf)
    rest = ~(nan | over)
    check(p.cpu()[rest], want[rest], err[rest], "fp32", "p")


@pytest.mark.parametrize("bits", [32, 8])
def test_squares_beyond_fp32(bits):
    """A finite gradient whose v is not one: nothing but the decay moves the parameter."""
    n = 1030
    gen = torch.Generator().manual_seed(1)
    p = torch.randn(n, generator=gen, dtype=torch.float32).cuda()
    g = torch.randn(n, generator=gen, dtype=torch.float32).cuda()
    for i, x in ((0, 1e25), (1, -1e22), (255, 1e20), (256, 5.8e19), (700, -5.9e19), (1024, 3e38), (1029, 1e25)):
        g[i] = x
    opt = AdamW([p], [g], LR, B1, B2, EPS, DECAY, bits)
    before = p.double().cpu()
    opt.step()
    zero = torch.zeros(n, dtype=torch.float64)
    m, v = _states(zero, zero, g.double().cpu())
    assert v[0] == v[700] == math.inf and v[256] < MOST
    _check_step(p, before, m, v, 1)
    if bits == 32:
        assert torch.equal(opt.v.cpu().double(), v) and torch.equal(opt.m.cpu().double(), m)
        g.normal_()
        before = p.double().cpu()
        opt.step()
        m, v = _states(m, v, g.double().cpu())
        assert v[0] == math.inf
        _check_step(p, before, m, v, 2)


def test_states_that_are_not_finite():
    """m and v of every kind side by side, fp32: what the formula gives, NaN where that is NaN."""
    kinds = [0.0, 1.0, 1e-30, 3e38, math.inf, -math.inf, math.nan]
    m = torch.tensor([x for x in kinds for _ in kinds], dtype=torch.float32)
    v = torch.tensor([x for _ in kinds for x in kinds], dtype=torch.float32)
    for value in (0.0, 0.25, 1e25, -3e38):
        p = torch.full_like(m, 0.5).cuda()
        g = torch.full_like(m, value).cuda()
        opt = AdamW([p], [g], LR, B1, B2, EPS, DECAY)
        opt.m.copy_(m), opt.v.copy_(v)
        before = p.double().cpu()
        opt.step()
        _check_step(p, before, *_states(m.double(), v.double(), g.double().cpu()), 1)


@pytest.mark.parametrize("bits", [32, 8])
def test_words_beside_the_tensors(bits):
    """Count, factor, flag and norms in the elements between parameters and gradients of one
    buffer: taken as others, one element further refused."""
    n = 300
    flat = torch.zeros(3 * n + 8, dtype=torch.float32, device="cuda")
    ints = flat.view(torch.int32)
    gen = torch.Generator().manual_seed(2)
    start, grad = (torch.randn(n, generator=gen, dtype=torch.float32).cuda() for _ in range(2))
    # coef | p | step, skip | g | norm words
    p, g = flat[1:1 + n], flat[n + 3:2 * n + 3]
    coef, step, skip = flat[0:1], ints[n + 1:n + 2], ints[n + 2:n + 3]
    p.copy_(start), g.copy_(grad), coef.fill_(0.5)
    table = pigan.TensorTable([g], [p], bits=bits)
    pigan.adamw_update(table, LR, B1, B2, EPS, coef=coef, step=step, skip=skip)
    want = start.clone()
    other = AdamW([want], [grad], LR, B1, B2, EPS, state_bits=bits)
    other.step(0.5)
    assert torch.equal(p, want) and torch.equal(g, grad) and step.item() == 1
    assert (coef.item(), skip.item()) == (0.5, 0) and not flat[2 * n + 3:].any()
    for bad in (dict(coef=flat[1:2]), dict(coef=flat[n:n + 1]), dict(skip=ints[n:n + 1]), dict(step=ints[1:2]),
                dict(step=ints[n + 3:n + 4]), dict(coef=coef, step=coef.view(torch.int32))):
        with pytest.raises(pigan.PiganError):
            pigan.adamw_update(table, LR, B1, B2, EPS, 1, **bad)
    assert torch.equal(p, want) and step.item() == 1


@pytest.mark.parametrize("bits", [32, 8])
def test_tensors_of_no_elements(bits):
    """A network's tensors may all be empty: every call is valid and changes nothing."""
    p, g = (torch.empty((0, 3), dtype=torch.float32, device="cuda") for _ in range(2))
    for n in (1, 3):
        opt = AdamW([p] * n, [g] * n, LR, state_bits=bits, capturable=True)
        norm, coef, flag = opt.grad_norm(0.5, 0.25)
        assert (norm.item(), coef.item(), flag.item()) == (0.0, 0.25, 0)
        opt.step(coef, flag)
        assert opt.t == 1
        m, v = opt.states()
        assert m.shape == v.shape == (0,) and m.dtype == v.dtype == torch.float32

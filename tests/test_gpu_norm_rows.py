"""Layer norm of rows whose rounded mean is off, and row loops of more than one
turn in every variant."""
import math

import pytest
import torch

from paper_1910_13444_amd import pigan
from _layers import DT, EPS32, act64, check, matrix
from test_gpu_norm import _backward, _forward, _seed

pytestmark = pytest.mark.gpu

F32 = dict(device="cuda", dtype=torch.float32)


@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("N", [3, 100, 700, 1500, 3000, 8191, 16384, 30001, 100003])
def test_constant_rows(N, dtype):
    """A constant row normalises to beta whatever its value: the sum that gave the
    mean was rounded, the distances from the mean are one small number, whose sums
    are exact."""
    c = torch.tensor([7.3, -0.1, 1000.7, 1 / 3, 3e-5, 0.0], dtype=DT[dtype], device="cuda")
    beta = torch.linspace(-1, 1, N, **F32)
    y, mean, rstd = pigan.layer_norm(c[:, None].repeat(1, N), torch.full((N,), 1.5, **F32), beta, eps=1e-5)
    assert torch.equal(mean, c.float())
    assert torch.equal(y, beta.to(DT[dtype]).expand_as(y))
    assert ((rstd.double() * math.sqrt(1e-5) - 1).abs() <= 4 * EPS32).all()


# Three turns of every variant's row loop and a ragged rest.  Forward: 2048 blocks of
# 256 threads (512 of 1024), which hold 32, 8, 4, 4, 1, 1, 1 and 1 rows; backward: 256
# blocks of 1024 threads with 128, 32, 16, 16, 4, 2, 1 and 1 rows, but 768 of 256 threads
# with 4 rows for 16-bit rows of 65 to 128 pieces.  A piece is 8 columns in 16 bits, 4 in
# fp32.
FORWARD = [(131109, 3), (32805, 25), (16421, 63), (16421, 125), (4133, 250), (4133, 500), (1061, 1000), (1061, 2000)]
BACKWARD = [(65573, 5), (16421, 25), (8229, 63), (8229, 125), (2085, 250), (1061, 500), (549, 1000), (549, 2000)]


@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("tail", [0, 1])
@pytest.mark.parametrize("M,pieces", FORWARD)
def test_forward_turns(M, pieces, tail, dtype):
    """Rows of whole pieces, and rows that end inside one."""
    N = pieces * (4 if dtype == "fp32" else 8) - tail
    print(f"norm forward {M} x {N} {dtype}", flush=True)
    x, _, _, ga = _forward(_seed(M, N), None, M, N, dtype)
    y = pigan.layer_norm(x, ga)[0]
    pigan.layer_norm(x, ga, out=x)
    assert torch.equal(x, y)


@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("tail", [0, 1])
@pytest.mark.parametrize("M,pieces", BACKWARD)
def test_backward_turns(M, pieces, tail, dtype):
    """With a skip, without, and in place over dy and over the skip's cotangent."""
    N = pieces * (4 if dtype == "fp32" else 8) - tail
    print(f"norm backward {M} x {N} {dtype}", flush=True)
    dy, x, mean, rstd, ga, r, dx, dg, db = _backward(_seed(M, N), None, M, N, dtype, True)
    _backward(_seed(M, N), None, M, N, dtype, False)
    p, q = dy.clone(), r.clone()
    for o in (pigan.layer_norm_backward(p, x, mean, rstd, ga, add=r, dx=p),
              pigan.layer_norm_backward(dy, x, mean, rstd, ga, add=q, dx=q)):
        assert torch.equal(o[0], dx) and torch.equal(o[1], dg) and torch.equal(o[2], db)


def test_turns_of_rows_too_long_for_registers():
    """More rows than blocks: the last ones as by themselves (a row's results depend
    on it alone), and all of dx over dy."""
    M, N, last = 65536 + 5, 16385, 7
    gen = torch.Generator(device="cuda").manual_seed(3)
    x = torch.randn((M, N), generator=gen, dtype=torch.bfloat16, device="cuda")
    y, mean, rstd = pigan.layer_norm(x)
    for got, want in zip((y, mean, rstd), pigan.layer_norm(x[-last:])):
        assert torch.equal(got[-last:], want)
    add = x.roll(1, 0)
    want = [pigan.layer_norm_backward(y[k], x[k], mean[k], rstd[k], add=add[k], need_params=False)[0]
            for k in (slice(0, last), slice(M - last, M))]
    dx = pigan.layer_norm_backward(y, x, mean, rstd, add=add, need_params=False, dx=y)[0]
    assert torch.equal(dx[:last], want[0]) and torch.equal(dx[-last:], want[1])


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("pad", [0, 5])
def test_act_backward_turns(dtype, pad):
    """More pieces than threads in every group, as one long row and row by row, over
    dy and over the pre-activation."""
    G, M, N = 3, 2011, 3003
    gen = _seed(pad)
    dy = matrix(gen, G, M, N, dtype, ld=N + pad)
    pre = matrix(gen, G, M, N, dtype, scale=2.0, ld=N + pad)
    d, s = dy.double().cpu(), act64(pre.double().cpu(), "silu")[1]
    g = pigan.act_backward(dy, pre, "silu")
    check(g, d * s, d.abs() * 4e-6, dtype, "g")
    over = pre.clone()
    assert torch.equal(pigan.act_backward(dy, over, "silu", out=over), g)
    assert torch.equal(pigan.act_backward(dy, pre, "silu", out=dy), g)

"""Layer norm of rows whose rounded mean is off, and row loops of more than one
turn in every variant."""
import math

import pytest
import torch

from paper_1910_13444_amd import pigan
from _layers import DT, EPS32

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

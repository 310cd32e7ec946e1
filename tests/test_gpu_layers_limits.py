"""The linear layer and layer norm at the edges of their sizes: no rows, and
more blocks than one dimension of a launch holds."""
import pytest
import torch

from paper_1910_13444_amd import pigan
from _layers import DT

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("G", [None, 3])
def test_no_rows_and_only_dx(dtype, G):
    def empty(*shape):
        return torch.empty((*((G,) if G else ()), *shape), dtype=DT[dtype], device="cuda")

    dx, dw, db = pigan.linear_backward(empty(0, 24), empty(0, 40), empty(24, 40), need_dw=False, need_db=False)
    assert dx.shape[-2:] == (0, 40) and dw is None and db is None
    y, mean, rstd = pigan.layer_norm(empty(0, 50))
    dx, dgamma, dbeta = pigan.layer_norm_backward(empty(0, 50), empty(0, 50), mean, rstd, need_params=False)
    assert dx.shape == y.shape and dgamma is None and dbeta is None

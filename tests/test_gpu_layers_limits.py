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


def _whole_numbers(*shape, dtype=torch.bfloat16):
    """-4 .. 4: short sums of products are exact in every type"""
    gen = torch.Generator(device="cuda").manual_seed(5)
    return torch.randint(-4, 5, shape, generator=gen, device="cuda", dtype=torch.int8).to(dtype)


def test_no_rows_of_a_wide_layer():
    """More elements of dw than 32 per thread of 2^32: zeros all the same."""
    K, N = 8193, 16385
    dw = torch.full((N, K), 7.0, dtype=torch.float32, device="cuda")
    db = torch.full((N,), 7.0, dtype=torch.float32, device="cuda")
    empty = torch.empty((0, K), dtype=torch.bfloat16, device="cuda")
    pigan.linear_backward(torch.empty((0, N), dtype=torch.bfloat16, device="cuda"), empty,
                          torch.empty((N, K), dtype=torch.bfloat16, device="cuda"), need_dx=False, dw=dw, db=db)
    assert not dw.any() and not db.any()


@pytest.mark.parametrize("M", [1, 3])
def test_strips_beyond_one_dimension_of_a_launch(M):
    """2^24 strips of 4 columns by 256 threads and a few more."""
    K, N = 8, 2 ** 26 + 25
    x, w = _whole_numbers(M, K), _whole_numbers(N, K)
    y = pigan.linear(x, w)
    for m in range(M):
        assert torch.equal(y[m], (w.float() * x[m].float()).sum(1).bfloat16())


def test_column_sums_beyond_one_dimension_of_a_launch():
    """Sums of more than 2^26 columns: 32 of them by 1024 threads."""
    N = 2 ** 26 + 41
    dy, x = _whole_numbers(2, N), _whole_numbers(2, N).flip(1).contiguous()
    mean, rstd = torch.zeros(2, device="cuda"), torch.ones(2, device="cuda")
    _, dgamma, dbeta = pigan.layer_norm_backward(dy, x, mean, rstd, need_dx=False)
    assert torch.equal(dbeta, dy.float().sum(0)) and torch.equal(dgamma, (dy.float() * x.float()).sum(0))
    dbeta = pigan.linear_backward(dy, x[:, :1], _whole_numbers(N, 1), need_dx=False, need_dw=False)[2]
    assert torch.equal(dbeta, dy.float().sum(0))

"""Calls of the linear layer and layer norm at the edges of what they take, as
far as the host decides them (these run without a GPU)."""
import pytest

from paper_1910_13444_amd import pigan
from test_layers_abi import FAKE, K, N, _linear, _norm, needs_lib

NONE = (0, 0, 0)


@needs_lib
@pytest.mark.parametrize("dt", [0, 1, 2])
def test_no_rows_and_only_dx(dt):
    """An empty batch's dx has no elements, and an empty tensor's address is 0:
    there is nothing to do, and nothing wrong."""
    L = pigan.lib()
    a = _linear(dt=dt, m=0, x=(0, K, 0), g=(0, N, 0), dx=(0, K, 0), dw=0, db=0)
    assert L.pigan_linear_backward(a, None, 0, None) == pigan.OK
    a = _norm(dt=dt, m=0, x=(0, N, 0), dy=(0, N, 0), dx=(0, N, 0), mean=0, rstd=0, dgamma=0, dbeta=0)
    assert L.pigan_layer_norm_backward(a, None, 0, None) == pigan.OK


@needs_lib
@pytest.mark.parametrize("rows,ld,gs", [((1 << 24) + 1, 1 << 40, 16), ((1 << 24) + 1, 1 << 40, 1 << 46),
                                        ((1 << 31) - 1, 1 << 40, 1 << 46), ((1 << 23) + 1, 1 << 40, 1 << 40)])
def test_groups_whose_extent_passes_63_bits(rows, ld, gs):
    """(rows - 1) * ld wraps around: the group still does not fit its stride."""
    L = pigan.lib()
    far = (FAKE, ld, gs)
    assert L.pigan_layer_norm_forward(_norm(G=2, m=rows, x=far, y=far), None) == pigan.EINVAL
    assert L.pigan_linear_forward(_linear(G=2, m=rows, x=far, y=far), FAKE, 1 << 60, None) == pigan.EINVAL
    one = (FAKE, ld, 0)
    assert L.pigan_layer_norm_forward(_norm(m=1 << 6, x=one, y=one, eps=0.0), None) == pigan.EINVAL
    assert b"eps" in L.pigan_last_error()   # the strides themselves are in range

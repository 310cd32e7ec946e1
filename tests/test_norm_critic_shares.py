"""The cotangents of the critic's loss, on the host."""
import pytest
import torch

from paper_1910_13444_amd.norm_critic import _shares


@pytest.mark.parametrize("dtype,unit", [(torch.bfloat16, 2.0 ** -7), (torch.float16, 2.0 ** -10), (torch.float32, 2.0 ** -23)])
@pytest.mark.parametrize("n", [1, 2, 3, 7, 24, 512, 1000, 16384, 20000, 100003])
def test_shares_add_up(n, dtype, unit):
    """Each is a neighbour of scale / n, and their sum is the scale (in fp32 to one
    rounding of the share)."""
    for scale in (1.0, 2.0 ** (n.bit_length() - 1)):
        if dtype == torch.float16 and scale / n < 2.0 ** -14:
            continue
        w = _shares(n, scale, dtype).double()
        assert w.shape == (n,) and ((w * n / scale - 1).abs() <= unit).all()
        assert abs(w.sum().item() / scale - 1) <= (2.0 ** -24 if dtype == torch.float32 else 1e-12)

"""The residual critic's training step on large batches: the gradients that its
update sees."""
import pytest
import torch

from paper_1910_13444_amd.norm_critic import CriticTrainer
from test_gpu_norm_critic import TOL, _critic, _reference, _rel

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("S,B", [(16384, 16384), (20000, 30000)])
def test_gradients_of_large_batches(dtype, S, B):
    """Within the bounds of a stored tensor's rounding, however small a sample's
    share 1 / S is: fp16 holds 5 bits of what is a 512th of it."""
    c, gen = _critic(24, 32, 2, None, 1, "silu", dtype)
    fake = torch.randn((1, S, 24), generator=gen, dtype=torch.float32).to(c.dtype).cuda()
    real = (torch.randn((1, B, 24), generator=gen, dtype=torch.float32) * 0.5 + 1).to(c.dtype).cuda()
    dscore = torch.cat([torch.full((1, S, 1), 1 / S), torch.full((1, B, 1), -1 / B)], 1)
    _, grads, _ = _reference(c, torch.cat([fake, real], 1), dscore)
    CriticTrainer(c, lr=0.0).step(fake, real)
    for n, t in grads.items():
        if n not in ("b_out", "beta"):   # 0 in exact arithmetic: the cotangents summed, 1 and w_out times
            assert _rel(c.g[n], t) <= TOL[dtype], n

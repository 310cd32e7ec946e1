"""The layer-normalised residual critic, its operators together: scores and every
gradient against autograd in 64 bits on the host, and its training runs.

Tolerances, relative per tensor (root of the sum of squares): a stored tensor is
off by about 0.4 units (half the last place) in this norm, a gradient of a critic
of three blocks stands behind about 30 stored tensors, whose errors are
independent, and a norm or a slope may enlarge an error threefold: 3 * 0.4 *
sqrt(30) = 6.6 units, 2.6e-2 in bf16 and 3.2e-3 in fp16.  In fp32 the products'
sums count as well: 1e-5, the framework's bar."""
import math

import pytest
import torch

from paper_1910_13444_amd import norm_critic
from paper_1910_13444_amd.norm_critic import CriticTrainer, NormCritic
from _layers import DT

pytestmark = pytest.mark.gpu

TOL = {"fp32": 1e-5, "bf16": 2.6e-2, "fp16": 3.2e-3}


def _reference(critic, x, dscore):
    """(scores, gradients by name, snapshots' cotangent) in 64 bits, at the
    weights and snapshots as they are stored."""
    act = {"none": lambda a: a, "tanh": torch.tanh, "relu": torch.relu, "silu": torch.nn.functional.silu,
           "gelu": torch.nn.functional.gelu}[critic.act]
    p = {n: (critic.w[n] if n in critic.w else t).double().cpu().requires_grad_() for n, t in critic.p.items()}
    x = x.double().cpu().requires_grad_()

    def lin(a, w, b):
        return a @ p[w].transpose(1, 2) + p[b].unsqueeze(1)

    def norm(h, i):
        m = h.mean(-1, keepdim=True)
        xh = (h - m) * ((h - m).square().mean(-1, keepdim=True) + critic.eps) ** -0.5
        return xh * p[f"gamma{i}"].unsqueeze(1) + p[f"beta{i}"].unsqueeze(1)

    h = act(lin(x, "w_in", "b_in"))
    for i in range(critic.blocks):
        h = h + lin(act(lin(norm(h, i), f"w1_{i}", f"b1_{i}")), f"w2_{i}", f"b2_{i}")
    score = lin(norm(h, ""), "w_out", "b_out")
    (score * dscore.double().cpu()).sum().backward()
    return score.detach(), {n: t.grad for n, t in p.items()}, x.grad


def _rel(got, want):
    return ((got.double().cpu() - want).norm() / want.norm()).item()


def _critic(n_in, width, blocks, hidden, G, act, dtype):
    c = NormCritic(n_in, width, blocks, hidden, G, act, DT[dtype])
    gen = torch.Generator().manual_seed(7)
    for n, t in c.p.items():   # shifts and scales away from 0 and 1
        if not n.startswith("w"):
            t.add_((torch.randn(t.shape, generator=gen, dtype=torch.float32) * 0.1).cuda())
    return c, gen


@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("n_in,width,blocks,hidden,G,B,act",
                         [(40, 64, 2, None, 1, 33, "silu"), (133, 100, 3, 201, 2, 70, "tanh"), (64, 96, 1, 32, 5, 1, "gelu"),
                          (9, 17, 0, None, 1, 5, "none"), (1000, 512, 3, None, 1, 256, "silu")])
def test_scores_and_gradients(dtype, n_in, width, blocks, hidden, G, B, act):
    c, gen = _critic(n_in, width, blocks, hidden, G, act, dtype)
    x = torch.randn((G, B, n_in), generator=gen, dtype=torch.float32).to(DT[dtype]).cuda()
    dscore = torch.randn((G, B, 1), generator=gen, dtype=torch.float32).to(DT[dtype]).cuda()
    score, saved = c.forward(x)
    assert torch.equal(score, c.score(x))
    c.grads.fill_(math.nan)
    dx = c.backward(dscore, saved, need_dx=True)
    want, grads, dx_want = _reference(c, x, dscore)
    assert _rel(score, want) <= TOL[dtype]
    assert _rel(dx, dx_want) <= TOL[dtype]
    for n, t in grads.items():
        assert _rel(c.g[n], t) <= TOL[dtype], n


def test_training_follows_the_64_bit_gradients():
    """Ten updates in fp32 against Adam in 64 bits on the reference's gradients."""
    c, gen = _critic(50, 64, 2, None, 2, "silu", "fp32")
    fake = torch.randn((2, 24, 50), generator=gen, dtype=torch.float32).cuda()
    real = torch.randn((2, 40, 50), generator=gen, dtype=torch.float32).cuda() * 0.5 + 0.3
    t = CriticTrainer(c, lr=1e-3)
    names = list(c.p)
    m = {n: 0.0 for n in names}
    v = {n: 0.0 for n in names}
    dscore = torch.cat([torch.full((2, 24, 1), 1 / 24), torch.full((2, 40, 1), -1 / 40)], 1)
    for k in range(1, 11):
        want, grads, _ = _reference(c, torch.cat([fake, real], 1), dscore.cuda())
        before = {n: p.double().cpu() for n, p in c.p.items()}
        loss = t.step(fake, real)
        w = want.squeeze(-1)
        # the scores' errors, each 1e-5 of their size, do not cancel in the difference of their means
        assert ((loss.double().cpu() - (w[:, :24].mean(1) - w[:, 24:].mean(1))).abs() <= 1e-5 * w.abs().amax(1)).all()
        for n in names:
            m[n] = 0.5 * m[n] + 0.5 * grads[n]
            v[n] = 0.9 * v[n] + 0.1 * grads[n] ** 2
            step = 1e-3 * (m[n] / (1 - 0.5 ** k)) / ((v[n] / (1 - 0.9 ** k)).sqrt() + 1e-8)
            if n in ("b_out", "beta"):
                continue   # 0 in exact arithmetic: the scores' cotangents summed, 1 and w_out times
            # a small gradient's relative error, and so its step's, may be large: judged over the tensor
            assert (c.p[n].double().cpu() - (before[n] - step)).norm() <= 2e-3 * step.norm() + 1e-6 * before[n].norm(), n


def test_weights_stay_within_the_clip_and_copies_follow():
    c, gen = _critic(64, 64, 1, None, 1, "tanh", "bf16")
    t = CriticTrainer(c, lr=1e-2, clip=0.05)
    fake = torch.randn((1, 16, 64), generator=gen, dtype=torch.float32).cuda()
    real = fake + 1
    for _ in range(3):
        t.step(fake, real)
    assert c.matrices.abs().max().item() <= torch.tensor(0.05, dtype=torch.float32).item()
    assert torch.equal(c.low, c.matrices.to(torch.bfloat16))


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_command_lowers_the_loss(dtype, capsys):
    losses = norm_critic.main(["--workload", "c1", "--steps", "30", "--width", "128", "--blocks", "2", "--dtype", dtype])
    assert len(losses) == 30 and all(math.isfinite(v) for v in losses)
    assert losses[-1] < losses[0] - 0.1
    assert "ms per step" in capsys.readouterr().out


def test_refusals():
    for bad in (dict(n_in=0), dict(width=0), dict(blocks=-1), dict(hidden=0), dict(G=0), dict(act="sine"),
                dict(dtype=torch.float64)):
        with pytest.raises(ValueError):
            NormCritic(**{**dict(n_in=8, width=8, blocks=1), **bad})
    c = NormCritic(8, 8, 1)
    with pytest.raises(ValueError):
        c.forward(torch.zeros((1, 4, 9), dtype=torch.bfloat16, device="cuda"))

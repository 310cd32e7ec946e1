"""The critic with group norm and AdamW over its tensors: scores and gradients against
autograd in 64 bits, updates against the definition, runs of the command.  Tolerances
as for the layer-normalised critic (test_gpu_norm_critic.py)."""
import math

import pytest
import torch

from paper_1910_13444_amd import norm_critic, pigan
from paper_1910_13444_amd.norm_critic import CriticTrainer, NormCritic
from _layers import DT

pytestmark = pytest.mark.gpu

TOL = {"fp32": 1e-5, "bf16": 2.6e-2, "fp16": 3.2e-3}
ACT = {"none": lambda a: a, "tanh": torch.tanh, "relu": torch.relu, "silu": torch.nn.functional.silu,
       "gelu": torch.nn.functional.gelu}


def _reference(c, x, dscore):
    act, n = ACT[c.act], c.channel_groups
    p = {k: (c.w[k] if k in c.w else t).double().cpu().requires_grad_() for k, t in c.p.items()}
    x = x.double().cpu().requires_grad_()

    def lin(a, w, b):
        return a @ p[w].transpose(1, 2) + p[b].unsqueeze(1)

    def norm(h, i):
        q = h.unflatten(-1, (n, -1))
        m = q.mean(-1, keepdim=True)
        q = ((q - m) * ((q - m).square().mean(-1, keepdim=True) + c.eps) ** -0.5).flatten(-2)
        return act(q * p[f"gamma{i}"].unsqueeze(1) + p[f"beta{i}"].unsqueeze(1))

    h = act(lin(x, "w_in", "b_in"))
    for i in range(c.blocks):
        h = h + lin(act(lin(norm(h, i), f"w1_{i}", f"b1_{i}")), f"w2_{i}", f"b2_{i}")
    score = lin(norm(h, ""), "w_out", "b_out")
    (score * dscore.double().cpu()).sum().backward()
    return score.detach(), {k: t.grad for k, t in p.items()}, x.grad


def _rel(got, want):
    return ((got.double().cpu() - want).norm() / want.norm()).item()


def _critic(n_in, width, blocks, G, act, dtype, groups):
    c = NormCritic(n_in, width, blocks, None, G, act, DT[dtype], norm="group", channel_groups=groups)
    gen = torch.Generator().manual_seed(7)
    for n, t in c.p.items():
        if not n.startswith("w"):
            t.add_((torch.randn(t.shape, generator=gen, dtype=torch.float32) * 0.1).cuda())
    return c, gen


@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("n_in,width,blocks,G,B,act,groups",
                         [(40, 64, 2, 1, 33, "silu", 8), (133, 100, 3, 2, 70, "tanh", 5), (64, 96, 1, 5, 1, "gelu", 12),
                          (500, 512, 3, 1, 256, "silu", 32)])
def test_scores_and_gradients(dtype, n_in, width, blocks, G, B, act, groups):
    c, gen = _critic(n_in, width, blocks, G, act, dtype, groups)
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


@pytest.mark.parametrize("dtype,bits,max_norm", [("fp32", 32, None), ("bf16", 8, 0.01), ("fp16", 32, 0.01)])
def test_updates(dtype, bits, max_norm):
    """A first update by the critic's own gradients: m = g' / 2, v = g'^2 / 10, so each
    element moves by lr (g' / (|g'| + eps) + decay p), g' the clipped gradient."""
    c, gen = _critic(50, 64, 2, 2, "silu", dtype, 4)
    lr, decay = 1e-3, 0.1
    t = CriticTrainer(c, lr, optimizer="adamw", weight_decay=decay, state_bits=bits, max_norm=max_norm)
    fake = torch.randn((2, 24, 50), generator=gen, dtype=torch.float32).cuda()
    real = torch.randn((2, 40, 50), generator=gen, dtype=torch.float32).cuda() * 0.5 + 0.3
    before = {n: p.double().cpu() for n, p in c.p.items()}
    t.step(fake, real)
    scale = t._cotangent(24, 40)[1]
    g = c.grads.double().cpu() / scale
    norm = g.norm().item()
    factor = 1.0 if max_norm is None else min(1.0, max_norm / norm)
    assert max_norm is None or factor < 1
    for n, p in c.p.items():
        gn = c.g[n].double().cpu() / scale * factor
        step = lr * (gn / (gn.abs() + 1e-8) + (decay if n in c.w else 0.0) * before[n])
        # the stored m and v, and coef, are off by 2^-24 each
        assert ((p.double().cpu() - (before[n] - step)).abs() <= 2.0 ** -24 * before[n].abs() + 2.0 ** -21 * lr).all(), n
    if c.low is not None:
        assert torch.equal(c.low, c.matrices.to(DT[dtype]))
    for _ in range(3):
        t.step(fake, real)
    assert torch.isfinite(c.master).all() and t.opt.t == 4
    if c.low is not None:
        assert torch.equal(c.low, c.matrices.to(DT[dtype]))


def test_clipped_weights_and_their_copies():
    c, gen = _critic(64, 64, 1, 1, "tanh", "bf16", 8)
    t = CriticTrainer(c, lr=1e-2, clip=0.05, optimizer="adamw", state_bits=8)
    fake = torch.randn((1, 16, 64), generator=gen, dtype=torch.float32).cuda()
    for _ in range(3):
        t.step(fake, fake + 1)
    assert c.matrices.abs().max().item() <= torch.tensor(0.05, dtype=torch.float32).item()
    assert torch.equal(c.low, c.matrices.to(torch.bfloat16))


@pytest.mark.parametrize("bits", [8, 32])
def test_the_command_runs(bits, capsys):
    losses = norm_critic.main(["--workload", "c1", "--steps", "5", "--width", "64", "--blocks", "2", "--norm", "group",
                               "--channel-groups", "4", "--optimizer", "adamw", "--weight-decay", "0.01", "--max-norm", "1",
                               "--state-bits", str(bits)])
    assert len(losses) == 5 and all(math.isfinite(v) for v in losses)
    assert "ms per step" in capsys.readouterr().out


def test_a_step_in_a_graph():
    """The whole step captured: forward, gradients, their norm, the update."""
    c, gen = _critic(40, 64, 2, 1, "silu", "bf16", 8)
    x = torch.randn((1, 30, 40), generator=gen, dtype=torch.float32).bfloat16().cuda()
    d = torch.randn((1, 30, 1), generator=gen, dtype=torch.float32).bfloat16().cuda()
    names = list(c.p)

    def trainer():
        from paper_1910_13444_amd.train import AdamW
        return AdamW([c.p[n] for n in names], [c.g[n] for n in names], 1e-3, state_bits=8, capturable=True,
                     copies=[c.w.get(n) for n in names])

    start = c.master.clone()

    def step(opt):
        c.backward(d, c.forward(x)[1])
        norm, coef, flag = opt.grad_norm(0.1)
        opt.step(coef, flag)

    eager = trainer()
    for _ in range(4):
        step(eager)
    want = c.master.clone()
    c.master.copy_(start)
    c.refresh()
    opt = trainer()
    graph = pigan.StepGraph(lambda: step(opt))   # runs one
    for _ in range(3):
        graph.replay()
        torch.cuda.synchronize()
    assert torch.equal(c.master, want) and opt.count.item() == 4


def test_refusals():
    for bad in (dict(norm="batch"), dict(norm="group", channel_groups=3), dict(norm="group", channel_groups=0)):
        with pytest.raises(ValueError):
            NormCritic(8, 8, 1, **bad)
    c = NormCritic(8, 8, 1)
    for bad in (dict(optimizer="sgd"), dict(weight_decay=0.1), dict(state_bits=8), dict(max_norm=1.0),
                dict(optimizer="adamw", state_bits=4)):
        with pytest.raises(ValueError):
            CriticTrainer(c, **bad)

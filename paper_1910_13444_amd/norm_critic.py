"""A layer-normalised residual critic, and a run that trains one.

Batch norm couples the samples of a batch, whose scores and gradients a
Wasserstein critic takes one by one; layer norm is what takes its place.  The
critic here is G independent networks (one per subdomain) of

  h   = act(x W_in^T + b_in)
  h  += act(n W_1^T + b_1) W_2^T + b_2,  n = LN(h)      `blocks` times
  score = LN(h) w_out^T + b_out

with any sizes.  Host logic only: every product, norm, gradient and update runs
in libpigan.so kernels on the current stream.  Between the operators nothing is
launched: bias, activation and residual are the forward products' epilogues, an
activation's slope and a skip's cotangent those of the reverse ones, and each
parameter gradient is written to its place in one flat fp32 vector.  There is no
second-order reverse pass: the trainer bounds the weights by clipping, not by a
gradient penalty.

  python -m paper_1910_13444_amd.norm_critic --steps 50

trains it to tell a teacher generator's sensor snapshots from those of an
untrained one, and prints the loss and the time of a step.
"""
from __future__ import annotations

import argparse
import math
import time
from dataclasses import dataclass

import torch

from . import configs, pigan
from .inputs import make_inputs
from .train import Adam


@dataclass
class _Block:
    """What a block's reverse pass needs of its forward pass."""
    h: torch.Tensor
    mean: torch.Tensor
    rstd: torch.Tensor
    n: torch.Tensor
    u: torch.Tensor
    pre: torch.Tensor


class NormCritic:
    """G critics of `n_in` inputs, `blocks` residual blocks of `width` (inner
    width `hidden`), in `dtype`, with fp32 master weights in one flat vector."""

    def __init__(self, n_in: int, width: int, blocks: int, hidden: int | None = None, G: int = 1, act: str = "silu",
                 dtype: torch.dtype = torch.bfloat16, device="cuda", seed: int = 0, eps: float = 1e-5):
        if min(n_in, width, G) < 1 or blocks < 0 or (hidden is not None and hidden < 1):
            raise ValueError("n_in, width, hidden and G must be positive, blocks not negative")
        if dtype not in pigan.TORCH_DTYPES:
            raise ValueError(f"dtype must be fp32, bf16 or fp16, got {dtype}")
        if act not in pigan.ACTS:
            raise ValueError(f"unknown activation {act!r}: one of {', '.join(pigan.ACTS)}")
        self.G, self.n_in, self.blocks, self.act, self.dtype, self.eps = G, n_in, blocks, act, dtype, eps
        hid = hidden or width
        shapes = {"w_in": (G, width, n_in), "b_in": (G, width)}
        for i in range(blocks):
            shapes |= {f"gamma{i}": (G, width), f"beta{i}": (G, width), f"w1_{i}": (G, hid, width), f"b1_{i}": (G, hid),
                       f"w2_{i}": (G, width, hid), f"b2_{i}": (G, width)}
        shapes |= {"gamma": (G, width), "beta": (G, width), "w_out": (G, 1, width), "b_out": (G, 1)}
        # the matrices first, so that one cast makes every 16-bit copy
        names = sorted(shapes, key=lambda n: not n.startswith("w"))
        n_mat = sum(math.prod(shapes[n]) for n in names if n.startswith("w"))
        f32 = dict(dtype=torch.float32, device=device)
        total = sum(math.prod(s) for s in shapes.values())
        self.master, self.grads = torch.zeros(total, **f32), torch.zeros(total, **f32)
        self.matrices = self.master[:n_mat]
        self.low = None if dtype == torch.float32 else torch.empty(n_mat, dtype=dtype, device=device)
        self.p, self.g, self.w = {}, {}, {}
        at = 0
        for n in names:
            s = shapes[n]
            end = at + math.prod(s)
            self.p[n], self.g[n] = self.master[at:end].view(s), self.grads[at:end].view(s)
            if n.startswith("w"):
                self.w[n] = self.p[n] if self.low is None else self.low[at:end].view(s)
            at = end
        gen = torch.Generator().manual_seed(seed)
        for n, t in self.p.items():
            if n.startswith("w"):   # Glorot normal, as the package's other networks
                t.copy_(torch.randn(t.shape, generator=gen, dtype=torch.float32) * math.sqrt(2 / (t.shape[1] + t.shape[2])))
            elif n.startswith("gamma"):
                t.fill_(1.0)
        self.refresh()

    def refresh(self):
        """Casts the matrices of changed master weights."""
        if self.low is not None:
            self.low.copy_(self.matrices)

    def forward(self, x: torch.Tensor):
        """(score [G, B, 1], saved) of the snapshots x [G, B, n_in]."""
        p, w = self.p, self.w
        h, pre_in = pigan.linear(x, w["w_in"], p["b_in"], self.act, save_pre=True)
        saved = []
        for i in range(self.blocks):
            n, mean, rstd = pigan.layer_norm(h, p[f"gamma{i}"], p[f"beta{i}"], self.eps)
            u, pre = pigan.linear(n, w[f"w1_{i}"], p[f"b1_{i}"], self.act, save_pre=True)
            saved.append(_Block(h, mean, rstd, n, u, pre))
            h = pigan.linear(u, w[f"w2_{i}"], p[f"b2_{i}"], residual=h)
        n, mean, rstd = pigan.layer_norm(h, p["gamma"], p["beta"], self.eps)
        score = pigan.linear(n, w["w_out"], p["b_out"])
        return score, (x, pre_in, saved, h, mean, rstd, n)

    def score(self, x: torch.Tensor) -> torch.Tensor:
        """Scores [G, B, 1] alone: a block's tensors are dropped with it."""
        p, w = self.p, self.w
        h = pigan.linear(x, w["w_in"], p["b_in"], self.act)
        for i in range(self.blocks):
            n, _, _ = pigan.layer_norm(h, p[f"gamma{i}"], p[f"beta{i}"], self.eps)
            u = pigan.linear(n, w[f"w1_{i}"], p[f"b1_{i}"], self.act)
            h = pigan.linear(u, w[f"w2_{i}"], p[f"b2_{i}"], residual=h, out=h)
        n, _, _ = pigan.layer_norm(h, p["gamma"], p["beta"], self.eps, out=h)
        return pigan.linear(n, w["w_out"], p["b_out"])

    def backward(self, dscore: torch.Tensor, saved, need_dx: bool = False) -> torch.Tensor | None:
        """Writes every parameter's gradient into `grads`; returns the
        snapshots' cotangent (a generator's way in) when it is needed."""
        p, w, g = self.p, self.w, self.g
        x, pre_in, blocks, h, mean, rstd, n = saved
        dn, _, _ = pigan.linear_backward(dscore, n, w["w_out"], dw=g["w_out"], db=g["b_out"])
        dh, _, _ = pigan.layer_norm_backward(dn, h, mean, rstd, p["gamma"], dgamma=g["gamma"], dbeta=g["beta"])
        for i in reversed(range(self.blocks)):
            b = blocks[i]
            dpre, _, _ = pigan.linear_backward(dh, b.u, w[f"w2_{i}"], self.act, b.pre, dw=g[f"w2_{i}"], db=g[f"b2_{i}"])
            dn, _, _ = pigan.linear_backward(dpre, b.n, w[f"w1_{i}"], dw=g[f"w1_{i}"], db=g[f"b1_{i}"])
            dh, _, _ = pigan.layer_norm_backward(dn, b.h, b.mean, b.rstd, p[f"gamma{i}"], add=dh, dgamma=g[f"gamma{i}"],
                                                 dbeta=g[f"beta{i}"])
        g_in = dh if self.act == "none" else pigan.act_backward(dh, pre_in, self.act)
        return pigan.linear_backward(g_in, x, w["w_in"], need_dx=need_dx, dw=g["w_in"], db=g["b_in"])[0]


def _shares(n: int, scale: float, dtype: torch.dtype) -> torch.Tensor:
    """n values of dtype that add up to `scale`: scale / n each, or its two
    neighbours in turn.  Rounded alike they would all be off by the same part (up
    to 2^-9 in bf16), and with them the balance of two sums of different n."""
    v = scale / n
    if dtype == torch.float32:
        return torch.full((n,), v, dtype=dtype)
    digits, least = (8, -133) if dtype == torch.bfloat16 else (11, -24)
    unit = 2.0 ** max(math.frexp(v)[1] - digits, least)
    return (torch.arange(n + 1, dtype=torch.float64) * (v / unit)).round().diff().mul(unit).to(dtype)


class CriticTrainer:
    """Wasserstein updates of a NormCritic on batches of fake and real
    snapshots.  `clip` bounds every element of its matrices after an update
    (None: no bound); the norms' scales and all shifts are free."""

    def __init__(self, critic: NormCritic, lr: float = 1e-4, clip: float | None = None):
        self.critic, self.clip = critic, clip
        self.opt = Adam(critic.master, lr)
        self._cotangents = {}   # of the scores, by batch sizes

    def _cotangent(self, S: int, B: int) -> tuple[torch.Tensor, float]:
        """(dscore [G, S + B, 1], its scale) of the loss.  fp16 has fewer bits
        below 2^-14: there the shares of large batches are scaled to about 1."""
        if (S, B) not in self._cotangents:
            c = self.critic
            scale = 2.0 ** (min(S, B).bit_length() - 1) if c.dtype == torch.float16 else 1.0
            d = torch.cat([_shares(S, scale, c.dtype), -_shares(B, scale, c.dtype)])
            self._cotangents[S, B] = d.to(c.master.device)[:, None].repeat(c.G, 1, 1), scale
        return self._cotangents[S, B]

    def step(self, fake: torch.Tensor, real: torch.Tensor) -> torch.Tensor:
        """One update; returns the loss mean D(fake) - mean D(real) per critic
        before it, [G], on the device."""
        c = self.critic
        S, B = fake.shape[1], real.shape[1]
        score, saved = c.forward(torch.cat([fake, real], 1).to(c.dtype))
        dscore, scale = self._cotangent(S, B)
        c.backward(dscore, saved)
        if scale != 1.0:
            c.grads.mul_(1.0 / scale)
        self.opt.step(c.grads)
        if self.clip is not None:
            c.matrices.clamp_(-self.clip, self.clip)
        c.refresh()
        s = score.float().squeeze(-1)
        return s[:, :S].mean(1) - s[:, S:].mean(1)


def snapshots(wl, params, z: torch.Tensor, xsY: torch.Tensor, xsU: torch.Tensor) -> torch.Tensor:
    """[G, S, n_sY + n_sU]: a generator's Y and u at the sensors, fp32."""
    y, u = (pigan.gen_forward(p, wl.gen_shape(), wl.d, z, xs, 0, dtype=wl.dtype, x_shared=True)[:, 0]
            for p, xs in zip(params, (xsY, xsU)))
    return torch.cat([y, u], -1)


def main(argv=None) -> list[float]:
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    ap.add_argument("--workload", default="c2", help="a paired-generator workload of configs.py")
    ap.add_argument("--width", type=int, default=512)
    ap.add_argument("--blocks", type=int, default=3)
    ap.add_argument("--act", default="silu", choices=sorted(pigan.ACTS))
    ap.add_argument("--dtype", default="bf16", choices=sorted(pigan.DTYPES))
    ap.add_argument("--steps", type=int, default=50)
    ap.add_argument("--lr", type=float, default=1e-4)
    ap.add_argument("--clip", type=float, default=None)
    a = ap.parse_args(argv)
    wl = configs.get(a.workload)
    if wl.trunk_gen or wl.is_hier:
        ap.error(f"--workload {a.workload}: a workload with one pair of generators per group is needed")
    inp = make_inputs(wl)
    dev = {k: torch.from_numpy(getattr(inp, k)).cuda() for k in ("pY", "pU", "tY", "tU", "z", "z_teach", "xsY", "xsU")}
    fake = snapshots(wl, (dev["pY"], dev["pU"]), dev["z"], dev["xsY"], dev["xsU"])
    real = snapshots(wl, (dev["tY"], dev["tU"]), dev["z_teach"], dev["xsY"], dev["xsU"])
    dtype = next(t for t, d in pigan.TORCH_DTYPES.items() if d == pigan.DTYPES[a.dtype])
    critic = NormCritic(fake.shape[-1], a.width, a.blocks, G=wl.G, act=a.act, dtype=dtype)
    trainer = CriticTrainer(critic, a.lr, a.clip)
    losses = []
    t0 = None
    for k in range(a.steps):
        losses.append(trainer.step(fake, real))
        if k == 0:
            torch.cuda.synchronize()
            t0 = time.perf_counter()
    torch.cuda.synchronize()
    losses = [v.mean().item() for v in losses]
    for k in range(0, a.steps, max(1, a.steps // 10)):
        print(f"step {k:4d}  loss {losses[k]:.5f}")
    if a.steps > 1:
        print(f"{wl.G} x [{fake.shape[1]} + {real.shape[1]}, {critic.n_in}] snapshots, width {a.width}, {a.blocks} blocks, "
              f"{a.dtype}: loss {losses[0]:.5f} -> {losses[-1]:.5f}, "
              f"{(time.perf_counter() - t0) / (a.steps - 1) * 1e3:.3f} ms per step")
    return losses


if __name__ == "__main__":
    main()

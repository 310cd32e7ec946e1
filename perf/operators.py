"""Layer norm and the fused linear layer: what is timed, and their plain forms.

The operators are the parts of a normalised residual network as a critic or a
generator trunk of this package uses it:

  linear_fwd   y = act(x w^T + bias) + residual, optionally with the
               pre-activation x w^T + bias as a second output
  linear_bwd   dx = (g w) act'(pre) + add,  dw = g^T x,  db = sum_rows g, where
               g is the cotangent of the layer's pre-activation and pre the
               pre-activation that x was formed from (the layer below's)
  act_bwd      g = dy act'(pre): a network's last activation
  norm_fwd     y = (x - mean) rstd gamma + beta over every row, with its mean
               and rstd = 1 / sqrt(variance + eps)
  norm_bwd     dx = rstd (h - mean_row(h) - xhat mean_row(h xhat)) + add,
               h = dy gamma; dgamma = sum_rows dy xhat, dbeta = sum_rows dy

Matrices are stored in the case's dtype; bias, gamma, beta, mean and rstd and
the parameter gradients are fp32.

A case is a dict of plain values:
  kind       one of the names above
  dtype      fp32 | bf16 | fp16
  G          groups: independent layers of one shape (subdomain critics)
  M, K, N    rows per group, inputs and outputs (norms and act_bwd: N columns)
  act        none | tanh | relu | gelu | silu
  res        a residual (linear_fwd), or a cotangent that is added to dx
  pre        linear_fwd: the pre-activation is stored too
  pad        elements between the end of a row and the next row
"""
from __future__ import annotations

import math

import torch

own = False

DT = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}
KINDS = ("linear_fwd", "linear_bwd", "act_bwd", "norm_fwd", "norm_bwd")
ACTS = ("none", "tanh", "relu", "gelu", "silu")
EPS = 1e-5


def _case(name=None, **kw):
    c = dict(kind="linear_fwd", dtype="bf16", G=1, M=1024, K=1024, N=1024, act="none", res=False, pre=False, pad=0)
    c.update(kw)
    if name is not None:
        c["name"] = name
    return c


def listed():
    return [
        # the first layer of the 5 x 2048 critic on ONE snapshot of 4096 + 4096 sensors: scoring a sample as it comes
        _case("fwd_one_snapshot", M=1, K=8192, N=2048, act="tanh"),
        # the thousand-sensor critic's first layer on a batch of 512 + 512 snapshots, kept for the reverse pass
        _case("fwd_critic_batch", M=1024, K=2000, N=1024, act="gelu", pre=True),
        # second layer of a residual block, width 1024, on collocation rows of a training step
        _case("fwd_block_rows", M=262144, K=1024, N=1024, res=True),
        # the reverse pass of that block's inner layer: activation below, on the rows of a chunk
        _case("bwd_block_rows", kind="linear_bwd", M=131072, K=1024, N=1024, act="gelu"),
        # 1 + 4 + 16 subdomain critics, 3 x 256, on 512 snapshots each, reverse pass of a hidden layer
        _case("bwd_subdomains", kind="linear_bwd", dtype="fp16", G=21, M=512, K=256, N=256, act="tanh"),
        # odd counts in fp32: a validation run's critic with 997 + 1003 sensors
        _case("bwd_odd_fp32", kind="linear_bwd", dtype="fp32", M=1001, K=2000, N=513, act="tanh"),
        # the last activation of the 1-D toy's critic, 64 generated and 64 real snapshots: a first run, a unit test
        _case("act_bwd_toy", kind="act_bwd", dtype="fp32", M=128, N=32, act="tanh"),
        # the last activation of a field network
        _case("act_bwd_rows", kind="act_bwd", M=65536, N=1024, act="silu"),
        # norm of a critic's batch of 1000 + 1000 sensor values, an odd batch
        _case("norm_fwd_critic", kind="norm_fwd", dtype="fp16", M=1023, N=2000),
        # norm in front of a residual block, width 512, collocation rows
        _case("norm_fwd_rows", kind="norm_fwd", M=262144, N=512),
        # its reverse pass with the block's skip cotangent, width 1024
        _case("norm_bwd_rows", kind="norm_bwd", M=131072, N=1024, res=True),
        # the reverse pass of a norm over whole snapshots of 8192 sensors
        _case("norm_bwd_snapshots", kind="norm_bwd", dtype="fp32", M=2048, N=8191),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


#: operations and bytes of the largest listed case: no drawn case costs more
MOST_FLOPS = 2.0 * 2 * 131072 * 1024 * 1024
MOST_BYTES = 2.0 * 3 * 262144 * 1024


def draw(rng):
    while True:
        kind = rng.choice(KINDS)
        c = _case(kind=kind, dtype=rng.choice(("bf16", "bf16", "fp16", "fp32")), G=rng.choice((1, 1, 1, 4, 16)),
                  M=_log(rng, 1, 262144), K=_log(rng, 8, 8192), N=_log(rng, 8, 8192), act=rng.choice(ACTS),
                  res=rng.random() < 0.4, pre=rng.random() < 0.5, pad=rng.choice((0, 0, 0, 8, 3)))
        if rng.random() < 0.6:   # most widths are whole multiples of 16
            c["K"], c["N"] = -(-c["K"] // 16) * 16, -(-c["N"] // 16) * 16
        if not kind.startswith("linear"):
            c["K"] = c["N"]
        if kind != "linear_fwd":
            c["pre"] = False
        if kind == "act_bwd":
            c["res"] = False
            c["act"] = rng.choice(ACTS[1:])
        if kind.startswith("norm"):
            c["act"] = "none"
            if kind == "norm_fwd":
                c["res"] = False
        w = work(c)
        # fp32 products cost about ten times those of 16 bits
        if w["flops"] * (10 if c["dtype"] == "fp32" else 1) <= MOST_FLOPS and w["bytes"] <= MOST_BYTES:
            return c


def work(case):
    G, M, K, N = case["G"], case["M"], case["K"], case["N"]
    e = 4 if case["dtype"] == "fp32" else 2
    kind, act, res = case["kind"], case["act"] != "none", bool(case["res"])
    if kind == "linear_fwd":
        b = e * (M * K + N * K + M * N * (1 + res + bool(case["pre"]))) + 4 * N
        f = 2.0 * M * N * K
    elif kind == "linear_bwd":
        b = e * (M * N + M * K * (2 + act + res) + N * K) + 4 * (N * K + N)
        f = 4.0 * M * N * K
    elif kind == "act_bwd":
        b, f = 3 * e * M * N, 10.0 * M * N
    elif kind == "norm_fwd":
        b, f = 2 * e * M * N + 8 * M + 8 * N, 8.0 * M * N
    else:
        b, f = e * M * N * (3 + res) + 8 * M + 12 * N, 14.0 * M * N
    return {"bytes": float(G * b), "flops": float(G * f)}


# ---------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------

def prepare(case, seed):
    dev, dt = "cuda", DT[case["dtype"]]
    gen = torch.Generator(device=dev)
    gen.manual_seed(int(seed))
    G, M, K, N, pad = case["G"], case["M"], case["K"], case["N"], case["pad"]

    def normal(rows, cols, scale=1.0, shift=0.0, padded=True):
        """[G, rows, cols] (no group axis for one group), rows `pad` elements apart"""
        p = pad if padded else 0
        t = torch.empty((G, rows, cols + p), dtype=dt, device=dev).normal_(0.0, 1.0, generator=gen)
        t = t.mul_(scale)
        if shift:
            t = t.add_(shift)
        t = t[..., :cols]
        return t if G > 1 else t[0]

    def vector(cols, scale, shift=0.0):
        t = torch.randn((G, cols), dtype=torch.float32, device=dev, generator=gen) * scale + shift
        return t if G > 1 else t[0]

    s = {"case": case, "act": case["act"]}
    kind = case["kind"]
    if kind == "linear_fwd":
        s |= {"x": normal(M, K), "w": normal(N, K, 1.0 / math.sqrt(K), padded=False), "bias": vector(N, 0.1),
              "residual": normal(M, N) if case["res"] else None}
    elif kind == "linear_bwd":
        s |= {"g": normal(M, N, 0.05), "x": normal(M, K), "w": normal(N, K, 1.0 / math.sqrt(K), padded=False),
              "pre": normal(M, K) if case["act"] != "none" else None,
              "add": normal(M, K, 0.05) if case["res"] else None}
    elif kind == "act_bwd":
        s |= {"dy": normal(M, N, 0.05), "pre": normal(M, N)}
    else:
        # sensor values and activations: a mean that is not zero
        s |= {"x": normal(M, N, 1.0, 0.5), "gamma": vector(N, 0.1, 1.0), "beta": vector(N, 0.1)}
        if kind == "norm_bwd":
            x = s["x"].float()
            mean = x.mean(-1)
            var = (x - mean[..., None]).square().mean(-1)
            s |= {"dy": normal(M, N, 0.05), "mean": mean, "rstd": (var + EPS).rsqrt(),
                  "add": normal(M, N, 0.05) if case["res"] else None}
    return s


# ---------------------------------------------------------------------------
# plain forms: elementary operations in fp32, rounded once at the end
# ---------------------------------------------------------------------------

def _act(a, act):
    if act == "tanh":
        return torch.tanh(a)
    if act == "relu":
        return a.clamp(min=0)
    if act == "gelu":
        return 0.5 * a * (1 + torch.erf(a * math.sqrt(0.5)))
    if act == "silu":
        return a * torch.sigmoid(a)
    return a


def _dact(a, act):
    if act == "tanh":
        return 1 - torch.tanh(a).square()
    if act == "relu":
        return (a > 0).to(a.dtype)
    if act == "gelu":
        return 0.5 * (1 + torch.erf(a * math.sqrt(0.5))) + a * torch.exp(-0.5 * a * a) * (1 / math.sqrt(2 * math.pi))
    sg = torch.sigmoid(a)
    return sg * (1 + a * (1 - sg))


def _plain(s):
    kind, act = s["case"]["kind"], s["act"]
    if kind == "linear_fwd":
        x, dt = s["x"], s["x"].dtype
        a = torch.matmul(x.float(), s["w"].float().transpose(-1, -2)) + s["bias"].unsqueeze(-2)
        y = _act(a, act)
        if s["residual"] is not None:
            y = y + s["residual"].float()
        return {"y": y.to(dt), "pre": a.to(dt)} if s["case"]["pre"] else {"y": y.to(dt)}
    if kind == "linear_bwd":
        g, x, w, dt = s["g"].float(), s["x"].float(), s["w"].float(), s["x"].dtype
        dx = torch.matmul(g, w)
        if s["pre"] is not None:
            dx = dx * _dact(s["pre"].float(), act)
        if s["add"] is not None:
            dx = dx + s["add"].float()
        return {"dx": dx.to(dt), "dw": torch.matmul(g.transpose(-1, -2), x), "db": g.sum(-2)}
    if kind == "act_bwd":
        return {"g": (s["dy"].float() * _dact(s["pre"].float(), act)).to(s["dy"].dtype)}
    x, dt, gamma = s["x"].float(), s["x"].dtype, s["gamma"].unsqueeze(-2)
    if kind == "norm_fwd":
        mean = x.mean(-1, keepdim=True)
        xc = x - mean
        rstd = (xc.square().mean(-1, keepdim=True) + EPS).rsqrt()
        y = xc * rstd * gamma + s["beta"].unsqueeze(-2)
        return {"y": y.to(dt), "mean": mean.squeeze(-1), "rstd": rstd.squeeze(-1)}
    dy, rstd = s["dy"].float(), s["rstd"].unsqueeze(-1)
    xhat = (x - s["mean"].unsqueeze(-1)) * rstd
    h = dy * gamma
    dx = rstd * (h - h.mean(-1, keepdim=True) - xhat * (h * xhat).mean(-1, keepdim=True))
    if s["add"] is not None:
        dx = dx + s["add"].float()
    return {"dx": dx.to(dt), "dgamma": (dy * xhat).sum(-2), "dbeta": dy.sum(-2)}


def run(state):
    if not own:
        return _plain(state)
    from paper_1910_13444_amd import pigan
    s, kind = state, state["case"]["kind"]
    if kind == "linear_fwd":
        if s["case"]["pre"]:
            y, pre = pigan.linear(s["x"], s["w"], s["bias"], act=s["act"], residual=s["residual"], save_pre=True)
            return {"y": y, "pre": pre}
        return {"y": pigan.linear(s["x"], s["w"], s["bias"], act=s["act"], residual=s["residual"])}
    if kind == "linear_bwd":
        dx, dw, db = pigan.linear_backward(s["g"], s["x"], s["w"], act=s["act"], pre=s["pre"], add=s["add"])
        return {"dx": dx, "dw": dw, "db": db}
    if kind == "act_bwd":
        return {"g": pigan.act_backward(s["dy"], s["pre"], s["act"])}
    if kind == "norm_fwd":
        y, mean, rstd = pigan.layer_norm(s["x"], s["gamma"], s["beta"], eps=EPS)
        return {"y": y, "mean": mean, "rstd": rstd}
    dx, dgamma, dbeta = pigan.layer_norm_backward(s["dy"], s["x"], s["mean"], s["rstd"], s["gamma"], add=s["add"])
    return {"dx": dx, "dgamma": dgamma, "dbeta": dbeta}


# ---------------------------------------------------------------------------
# the definitions in 64 bits
# ---------------------------------------------------------------------------

def _value64(a, act):
    """(act(a), act'(a)) in 64 bits"""
    one = torch.ones_like(a)
    if act == "tanh":
        return a.tanh(), 1 / a.cosh().square()
    if act == "relu":
        pos = torch.where(a > 0, one, torch.zeros_like(a))
        return a * pos, pos
    if act == "gelu":
        cdf = 0.5 * torch.special.erfc(-a / math.sqrt(2.0))
        return a * cdf, cdf + a * torch.exp(-a * a / 2) / math.sqrt(2 * math.pi)
    if act == "silu":
        e = 1 / (1 + torch.exp(-a))
        return a * e, e + a * e * (1 - e)
    return a, one


def exact(case, seed):
    s = prepare(case, seed)
    kind, act = case["kind"], case["act"]
    v = {k: t.double() if t.dim() != 0 else t for k, t in s.items() if isinstance(t, torch.Tensor)}
    if case["G"] == 1:   # a group axis everywhere
        v = {k: t[None] for k, t in v.items()}
    out = []
    for g in range(case["G"]):
        q = {k: t[g] for k, t in v.items()}
        if kind == "linear_fwd":
            a = torch.addmm(q["bias"][None, :], q["x"], q["w"].t().contiguous())
            y = _value64(a, act)[0]
            if "residual" in q:
                y = y + q["residual"]
            r = {"y": y, "pre": a} if case["pre"] else {"y": y}
        elif kind == "linear_bwd":
            dx = q["g"].mm(q["w"])
            if "pre" in q:
                dx = _value64(q["pre"], act)[1] * dx
            if "add" in q:
                dx = q["add"] + dx
            r = {"dx": dx, "dw": q["g"].t().contiguous().mm(q["x"]), "db": torch.sum(q["g"], 0)}
        elif kind == "act_bwd":
            r = {"g": _value64(q["pre"], act)[1] * q["dy"]}
        elif kind == "norm_fwd":
            var, mean = torch.var_mean(q["x"], 1, correction=0)
            rstd = 1 / torch.sqrt(var + EPS)
            r = {"y": (q["x"] - mean[:, None]) * rstd[:, None] * q["gamma"] + q["beta"], "mean": mean, "rstd": rstd}
        else:
            n = case["N"]
            xh = (q["x"] - q["mean"][:, None]) * q["rstd"][:, None]
            h = q["dy"] * q["gamma"][None, :]
            dx = h - h.sum(1, keepdim=True) / n - xh * ((h * xh).sum(1, keepdim=True) / n)
            dx = dx * q["rstd"][:, None]
            if "add" in q:
                dx = dx + q["add"]
            r = {"dx": dx, "dgamma": (q["dy"] * xh).sum(0), "dbeta": q["dy"].sum(0)}
        out.append(r)
    r = {k: torch.stack([o[k] for o in out]) for k in out[0]}
    return r if case["G"] > 1 else {k: t[0] for k, t in r.items()}

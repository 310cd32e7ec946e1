"""Group norm with an activation, the norm of many gradients and the AdamW step
over many tensors: what is timed, and their plain forms.

They are the rest of a normalised critic's training step beside its linear
layers:

  gn_fwd     over the P points and c = C / n channels of each of a sample's n
             channel groups: mean, rstd = 1 / sqrt(variance + eps),
             y = act((x - mean) rstd gamma + beta); channels last
  gn_bwd     from dy, with xh = (x - mean) rstd, da = dy act'(xh gamma + beta)
             and h = da gamma:  dx = rstd (h - mean(h) - xh mean(h xh)) + add,
             dgamma = sum of da xh and dbeta = sum of da over samples and points
  grad_norm  norm = scale sqrt(sum of all g^2), the factor
             coef = scale min(1, max_norm / norm), and whether norm is not finite
  adamw      g' = coef g,  m = b1 m + (1 - b1) g',  v = b2 v + (1 - b2) g'^2,
             p -= lr ((m / (1 - b1^t)) / (sqrt(v / (1 - b2^t)) + eps) + decay_i p),
             optionally behind grad_norm, with 16-bit copies of p

States in 8 bits are codes of blocks of 256 elements of a tensor (the last one
shorter) with an fp32 scale s, the largest size in the block:
  m = s q |q| / 127^2,  q = sign(m) round(127 sqrt(|m| / s))
  v = s q^4 / 255^4,    q = round(255 (v / s)^(1/4)), at least 1 for v > 0
where m and v are the new states as fp32 values; the update takes those, the
codes are what the next step finds.  A tensor's codes begin at a whole block.

Matrices are stored in the case's dtype; gamma, beta, mean, rstd, the parameter
gradients, p, m, v, the scales and coef are fp32.

A case is a dict of plain values:
  kind       one of the names above
gn_fwd, gn_bwd:
  dtype      fp32 | bf16 | fp16
  G          independent layers of one shape (subdomain critics)
  S, P, C    samples, points of a sample, channels
  n          channel groups
  act        none | tanh | relu | gelu | silu
  res        a cotangent is added to dx
  pad        elements between the end of a point's channels and the next point
grad_norm, adamw: the tensors of D networks of L layers of width W on n_in inputs
(a matrix and a vector each, and the output layer's)
  gdt        type of the gradients
  bits       of the states: 32 or 8
  copy       type of the copies of p: none | bf16 | fp16
  clip       grad_norm in front of the step
  scale      factor of all gradients (1 / loss scale)
"""
from __future__ import annotations

import math

import torch

own = False

DT = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}
ACTS = ("none", "tanh", "relu", "gelu", "silu")
EPS = 1e-5
LR, B1, B2, ADAM_EPS, DECAY, MAX_NORM = 1e-4, 0.5, 0.9, 1e-8, 0.01, 1.0
BLOCK = 256


def _gn(name=None, **kw):
    c = dict(kind="gn_fwd", dtype="bf16", G=1, S=1, P=1, C=128, n=8, act="none", res=False, pad=0)
    c.update(kw)
    if name is not None:
        c["name"] = name
    return c


def _opt(name=None, **kw):
    c = dict(kind="adamw", D=1, L=3, W=256, n_in=400, gdt="fp32", bits=32, copy="none", clip=False, scale=1.0)
    c.update(kw)
    if name is not None:
        c["name"] = name
    return c


def listed():
    return [
        # ONE sample's 64 sensors, 128 channels: scoring a snapshot as it comes
        _gn("gn_one_sample", S=1, P=64, C=128, n=8, act="silu"),
        # the 2-D workload's field: 256 samples of 1024 points, width 128
        _gn("gn_points", S=256, P=1024, C=128, n=16, act="silu"),
        # the rows of a critic's hidden layer, one point each, width 1024
        _gn("gn_rows", dtype="fp16", S=131072, P=1, C=1024, n=32),
        # fields on a grid of 256 x 256 points: a group is far more than a block of threads holds
        _gn("gn_grid", S=16, P=65536, C=128, n=8, act="gelu"),
        # reverse pass on the 2-D workload's points, width 256, with a block's skip cotangent
        _gn("gn_bwd_points", kind="gn_bwd", S=128, P=1024, C=256, n=32, act="silu", res=True),
        # odd counts in fp32: four subdomains, 1000 sensors, 24 groups of five channels
        _gn("gn_bwd_odd_fp32", kind="gn_bwd", dtype="fp32", G=4, S=21, P=1000, C=120, n=24, act="tanh"),
        # the gradients of the 5 x 2048 critic on 8192 sensors, fp32
        _opt("norm_critic", kind="grad_norm", L=5, W=2048, n_in=8192),
        # the gradients of 21 subdomain critics, 3 x 256, in bf16
        _opt("norm_subdomains", kind="grad_norm", D=21, n_in=80, gdt="bf16"),
        # the step of the 5 x 2048 critic with its 16-bit copies
        _opt("adamw_critic", L=5, W=2048, n_in=8192, copy="bf16"),
        # 273 subdomain critics, 3 x 256, 2184 tensors, clipped
        _opt("adamw_subdomains", D=273, n_in=20, clip=True),
        # the 21 x 1024 network with states in 8 bits, clipped, with copies
        _opt("adamw8_trunk", L=21, W=1024, n_in=130, bits=8, copy="bf16", clip=True),
        # the 1-D toy's critic: a first run, a unit test
        _opt("adamw8_toy", L=2, W=32, n_in=16, bits=8),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


#: bytes of the largest listed cases: no drawn case costs more
MOST_GN = 2.0 * 2 * 131072 * 1024
MOST_PARAMS = 273 * 137729


def _draw_gn(rng):
    while True:
        c = _gn(kind=rng.choice(("gn_fwd", "gn_bwd")), dtype=rng.choice(("bf16", "bf16", "fp16", "fp32")),
                G=rng.choice((1, 1, 1, 4)), S=_log(rng, 1, 131072), P=rng.choice((1, _log(rng, 1, 65536), _log(rng, 1, 65536))),
                C=_log(rng, 8, 2048), act=rng.choice(ACTS), pad=rng.choice((0, 0, 0, 8, 3)))
        if rng.random() < 0.6:   # most widths are whole multiples of 16
            c["C"] = -(-c["C"] // 16) * 16
        divisors = [k for k in range(1, c["C"] + 1) if c["C"] % k == 0 and c["P"] * c["C"] // k >= 8]
        if not divisors:
            continue
        c["n"] = rng.choice(divisors)
        if c["kind"] == "gn_bwd":
            c["res"] = rng.random() < 0.4
        if work(c)["bytes"] <= MOST_GN:
            return c


def _draw_opt(rng):
    while True:
        c = _opt(kind=rng.choice(("grad_norm", "adamw", "adamw")), D=rng.choice((1, _log(rng, 1, 273))), L=_log(rng, 1, 21),
                 W=_log(rng, 8, 2048), n_in=_log(rng, 5, 8192), gdt=rng.choice(("fp32", "fp32", "bf16", "fp16")),
                 copy=rng.choice(("none", "bf16", "fp16")), scale=rng.choice((1.0, 1.0, 2.0 ** -10)))
        if c["kind"] == "adamw":
            c["bits"] = rng.choice((32, 8))
            c["clip"] = rng.random() < 0.5
        else:
            c["copy"] = "none"
        if sum(_sizes(c)) <= MOST_PARAMS and len(_sizes(c)) <= 2200:
            return c


def draw(rng):
    return _draw_gn(rng) if rng.random() < 0.55 else _draw_opt(rng)


def _shapes(case):
    """shapes of the case's tensors, in the order of their places in the flat vectors"""
    W, one = case["W"], []
    for i in range(case["L"]):
        one += [(W, case["n_in"] if i == 0 else W), (W,)]
    return (one + [(1, W), (1,)]) * case["D"]


def _sizes(case):
    return [math.prod(s) for s in _shapes(case)]


def work(case):
    if case["kind"].startswith("gn"):
        e = 4 if case["dtype"] == "fp32" else 2
        N, stats = float(case["G"] * case["S"] * case["P"] * case["C"]), 8.0 * case["G"] * case["S"] * case["n"]
        if case["kind"] == "gn_fwd":
            return {"bytes": 2 * e * N + stats + 8.0 * case["G"] * case["C"], "flops": 10 * N}
        return {"bytes": (3 + bool(case["res"])) * e * N + stats + 16.0 * case["G"] * case["C"], "flops": 25 * N}
    N, e = float(sum(_sizes(case))), 4 if case["gdt"] == "fp32" else 2
    if case["kind"] == "grad_norm":
        return {"bytes": e * N + 12, "flops": 2 * N}
    # p is read and written; 8-bit states are read and written, and given as the values they stand for
    states = 16.0 if case["bits"] == 32 else 4 + 8 + 16.0 / BLOCK
    return {"bytes": N * (8 + e + states + (0 if case["copy"] == "none" else 2)), "flops": 20 * N}


# ---------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------

def _prepare_gn(case, gen):
    dev, dt = "cuda", DT[case["dtype"]]
    G, S, P, C, n = (case[k] for k in ("G", "S", "P", "C", "n"))

    def vector(scale, shift=0.0):
        t = torch.randn((G, C), dtype=torch.float32, device=dev, generator=gen) * scale + shift
        return t if G > 1 else t[0]

    def normal(scale, spread=None, shift=None):
        """[G, S, P, C] (no group axis for one group), points `pad` elements apart"""
        t = torch.empty((G, S, P, C + case["pad"]), dtype=dt, device=dev).normal_(0.0, 1.0, generator=gen)[..., :C]
        t.mul_(scale if spread is None else spread.to(dt))
        if shift is not None:
            t.add_(shift.to(dt))
        return t if G > 1 else t[0]

    # activations: channels of different means and spreads
    lift = torch.randn(C, dtype=torch.float32, device=dev, generator=gen) * 0.5 + 0.5
    spread = torch.rand(C, dtype=torch.float32, device=dev, generator=gen) + 0.5
    s = {"case": case, "x": normal(1.0, spread, lift), "gamma": vector(0.1, 1.0), "beta": vector(0.1)}
    if case["kind"] == "gn_bwd":
        x = s["x"].float().reshape(G, S, P, n, C // n)
        mean = x.mean((2, 4), keepdim=True)
        var = (x - mean).square().mean((2, 4))
        s |= {"mean": mean.reshape(G, S, n), "rstd": (var + EPS).rsqrt(), "dy": normal(0.05),
              "add": normal(0.05) if case["res"] else None}
        if G == 1:
            s["mean"], s["rstd"] = s["mean"][0], s["rstd"][0]
    return s


def _prepare_opt(case, gen):
    dev, f32 = "cuda", dict(dtype=torch.float32, device="cuda")
    shapes, sizes = _shapes(case), _sizes(case)
    n = sum(sizes)
    counts = torch.tensor(sizes, device=dev)
    # a tensor's gradients have a size of their own: 1e-6 to 1e-3
    size = torch.exp(math.log(1e-6) + math.log(1e3) * torch.rand(len(sizes), generator=gen, **f32)).repeat_interleave(counts)
    s = {"case": case, "t": 10, "p": torch.randn(n, generator=gen, **f32) * 0.05,
         "g": (torch.randn(n, generator=gen, **f32) * size / case["scale"]).clamp(-6e4, 6e4).to(DT[case["gdt"]])}

    def views(flat):
        return [t.view(sh) for t, sh in zip(flat.split(sizes), shapes)]

    if case["kind"] == "grad_norm":
        if own:
            from paper_1910_13444_amd import pigan
            s["table"] = pigan.TensorTable(grads=views(s["g"]))
        return s
    m = torch.randn(n, generator=gen, **f32) * size * 0.5
    v = (torch.randn(n, generator=gen, **f32) * size).square()
    decay = [DECAY if len(sh) == 2 else 0.0 for sh in shapes]
    s["decay"] = torch.tensor(decay, **f32).repeat_interleave(counts)
    s["low"] = None if case["copy"] == "none" else torch.empty(n, dtype=DT[case["copy"]], device=dev)
    if case["bits"] == 8:
        blocks = (counts + BLOCK - 1) // BLOCK
        first = (blocks.cumsum(0) - blocks) * BLOCK - (counts.cumsum(0) - counts)
        s["at"] = torch.arange(n, device=dev) + first.repeat_interleave(counts)   # an element's place among whole blocks
        s["places"] = int(blocks.sum()) * BLOCK
        pad = torch.zeros((2, s["places"]), dtype=torch.float64, device=dev)
        pad[0, s["at"]], pad[1, s["at"]] = m.double(), v.double()
        (s["m"], s["m_scale"]), (s["v"], s["v_scale"]) = _encode_m(pad[0]), _encode_v(pad[1])
    else:
        s["m"], s["v"] = m, v
    if own:
        from paper_1910_13444_amd import train
        opt = s["opt"] = train.AdamW(views(s["p"]), views(s["g"]), LR, B1, B2, ADAM_EPS, weight_decay=decay,
                                     state_bits=case["bits"], copies=None if s["low"] is None else views(s["low"]))
        opt.t = s["t"]
        opt.m.copy_(s["m"]), opt.v.copy_(s["v"])
        if case["bits"] == 8:
            opt.m_scale.copy_(s["m_scale"]), opt.v_scale.copy_(s["v_scale"])
    return s


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(int(seed))
    return _prepare_gn(case, gen) if case["kind"].startswith("gn") else _prepare_opt(case, gen)


# ---------------------------------------------------------------------------
# plain forms: elementary operations in fp32, rounded once at the end; the states
# in 8 bits, which round at borders, and long sums of squares in fp64
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


def _plain_gn(s):
    case, x, gamma, beta = s["case"], s["x"], s["gamma"], s["beta"]
    n, act, dt = case["n"], case["act"], x.dtype
    lead, (S, P, C) = x.shape[:-3], x.shape[-3:]
    wide = (*lead, 1, 1, n, C // n)
    xs, gamma, beta = x.float().reshape(*lead, S, P, n, C // n), gamma.reshape(wide), beta.reshape(wide)
    over = (-3, -1)
    if case["kind"] == "gn_fwd":
        mean = xs.mean(over, keepdim=True)
        xc = xs - mean
        rstd = (xc.square().mean(over, keepdim=True) + EPS).rsqrt()
        y = _act(xc * rstd * gamma + beta, act).to(dt)
        return {"y": y.reshape(x.shape), "mean": mean.reshape(*lead, S, n), "rstd": rstd.reshape(*lead, S, n)}
    rstd = s["rstd"].reshape(*lead, S, 1, n, 1)
    xh = (xs - s["mean"].reshape(*lead, S, 1, n, 1)) * rstd
    da = s["dy"].float().reshape(xs.shape)
    if act != "none":
        da = da * _dact(xh * gamma + beta, act)
    h = da * gamma
    dx = rstd * (h - h.mean(over, keepdim=True) - xh * (h * xh).mean(over, keepdim=True))
    dx = dx.reshape(x.shape)
    if s["add"] is not None:
        dx = dx + s["add"].float()
    return {"dx": dx.to(dt), "dgamma": (da * xh).sum((-4, -3)).reshape(*lead, C),
            "dbeta": da.sum((-4, -3)).reshape(*lead, C)}


def _encode_m(m):
    s = m.view(-1, BLOCK).abs().amax(1).float()
    q = (m.view(-1, BLOCK).abs() / torch.where(s > 0, s, 1.0).double()[:, None]).sqrt().mul(127).round().clamp(max=127)
    return (q.to(torch.int8) * m.view(-1, BLOCK).sign().to(torch.int8)).view(-1), s


def _encode_v(v):
    s = v.view(-1, BLOCK).amax(1).float()
    q = (v.view(-1, BLOCK) / torch.where(s > 0, s, 1.0).double()[:, None]).sqrt().sqrt().mul(255).round().clamp(max=255)
    return torch.where(v.view(-1, BLOCK) > 0, q.clamp(min=1), q).to(torch.uint8).view(-1), s


def _decode_m(q, s):
    q = q.view(-1, BLOCK).double()
    return (q * q.abs() * (s.double() / 127 ** 2)[:, None]).view(-1)


def _decode_v(q, s):
    return (q.view(-1, BLOCK).double().square().square() * (s.double() / 255 ** 4)[:, None]).view(-1)


def _plain_norm(g, scale):
    norm = scale * g.double().square().sum().sqrt()
    coef = scale * torch.where(norm > MAX_NORM, MAX_NORM / norm, 1.0)
    return {"norm": norm.float(), "coef": coef.float(), "nonfinite": (~torch.isfinite(norm)).to(torch.int32)}


def _plain_adamw(s):
    case = s["case"]
    s["t"] += 1
    c1, c2 = 1 / (1 - B1 ** s["t"]), 1 / (1 - B2 ** s["t"])
    out = _plain_norm(s["g"], case["scale"]) if case["clip"] else {}
    coef = out["coef"] if case["clip"] else case["scale"]
    p = s["p"]
    if case["bits"] == 32:
        g = s["g"].float() * coef
        m = s["m"].mul_(B1).add_((1 - B1) * g)
        v = s["v"].mul_(B2).add_((1 - B2) * g * g)
        p -= LR * (m * c1 / ((v * c2).sqrt() + ADAM_EPS) + s["decay"] * p)
        out |= {"m": m, "v": v}
    else:
        at = s["at"]
        g = torch.zeros(s["places"], dtype=torch.float64, device=p.device)
        g[at] = s["g"].double() * coef.double() if case["clip"] else s["g"].double() * coef
        m = (B1 * _decode_m(s["m"], s["m_scale"]) + (1 - B1) * g).float().double()
        v = (B2 * _decode_v(s["v"], s["v_scale"]) + (1 - B2) * g * g).float().double()
        u = m * c1 / ((v * c2).sqrt() + ADAM_EPS)
        p.copy_(p.double() - LR * (u[at] + s["decay"].double() * p.double()))
        (s["m"], s["m_scale"]), (s["v"], s["v_scale"]) = _encode_m(m), _encode_v(v)
        out |= {"m": _decode_m(s["m"], s["m_scale"]).float(), "v": _decode_v(s["v"], s["v_scale"]).float()}
    if s["low"] is not None:
        out["low"] = s["low"].copy_(p)
    return out | {"p": p}


def run(state):
    s, kind = state, state["case"]["kind"]
    if not own:
        return _plain_gn(s) if kind.startswith("gn") else _plain_adamw(s) if kind == "adamw" else _plain_norm(s["g"], s["case"]["scale"])
    from paper_1910_13444_amd import pigan
    c = s["case"]
    if kind == "gn_fwd":
        y, mean, rstd = pigan.group_norm(s["x"], c["n"], s["gamma"], s["beta"], act=c["act"], eps=EPS)
        return {"y": y, "mean": mean, "rstd": rstd}
    if kind == "gn_bwd":
        dx, dgamma, dbeta = pigan.group_norm_backward(s["dy"], s["x"], s["mean"], s["rstd"], s["gamma"], s["beta"],
                                                      act=c["act"], add=s["add"])
        return {"dx": dx, "dgamma": dgamma, "dbeta": dbeta}
    if kind == "grad_norm":
        norm, coef, nonfinite = pigan.grad_norm(s["table"], max_norm=MAX_NORM, scale=c["scale"])
        return {"norm": norm, "coef": coef, "nonfinite": nonfinite}
    opt, out = s["opt"], {}
    if c["clip"]:
        norm, coef, nonfinite = opt.grad_norm(max_norm=MAX_NORM, scale=c["scale"])
        opt.step(scale=coef, skip=nonfinite)
        out = {"norm": norm, "coef": coef, "nonfinite": nonfinite}
    else:
        opt.step(scale=c["scale"])
    m, v = opt.states()
    out |= {"m": m, "v": v, "p": s["p"]}
    if s["low"] is not None:
        out["low"] = s["low"]
    return out


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


def _exact_gn(case, s):
    G, S, P, C, n = (case[k] for k in ("G", "S", "P", "C", "n"))
    c = C // n
    shape = (G, S, P, C)
    x, gamma, beta = s["x"].reshape(shape), s["gamma"].reshape(G, C).double(), s["beta"].reshape(G, C).double()
    backward = case["kind"] == "gn_bwd"
    outs = [torch.empty((G, S, P, C), dtype=torch.float64, device=x.device)]
    outs += [torch.zeros((G, C), dtype=torch.float64, device=x.device) for _ in range(2)] if backward else \
            [torch.empty((G, S, n), dtype=torch.float64, device=x.device) for _ in range(2)]
    if backward:
        dy = s["dy"].reshape(shape)
        add = None if s["add"] is None else s["add"].reshape(shape)
        stats = [s[k].reshape(G, S, n).double() for k in ("mean", "rstd")]
    some = max(1, (1 << 24) // (P * C))   # samples at a time
    for g in range(G):
        for i in range(0, S, some):
            part = slice(i, i + some)
            q = x[g, part].double().unflatten(-1, (n, c)).permute(0, 2, 1, 3).reshape(-1, n, P * c)   # a group's values in a row
            ga = gamma[g].view(n, 1, c).expand(n, P, c).reshape(n, P * c)
            be = beta[g].view(n, 1, c).expand(n, P, c).reshape(n, P * c)

            def back(t):
                return t.view(-1, n, P, c).permute(0, 2, 1, 3).reshape(-1, P, C)

            if not backward:
                var, mean = torch.var_mean(q, -1, correction=0)
                rstd = 1 / torch.sqrt(var + EPS)
                outs[0][g, part] = back(_value64((q - mean[..., None]) * rstd[..., None] * ga + be, case["act"])[0])
                outs[1][g, part], outs[2][g, part] = mean, rstd
                continue
            mean, rstd = stats[0][g, part, :, None], stats[1][g, part, :, None]
            xh = (q - mean) * rstd
            d = dy[g, part].double().unflatten(-1, (n, c)).permute(0, 2, 1, 3).reshape(-1, n, P * c)
            d = _value64(xh * ga + be, case["act"])[1] * d
            h = d * ga
            dx = back(rstd * (h - h.sum(-1, keepdim=True) / (P * c) - xh * ((h * xh).sum(-1, keepdim=True) / (P * c))))
            outs[0][g, part] = dx if add is None else dx + add[g, part].double()
            outs[1][g] += back(d * xh).sum((0, 1))
            outs[2][g] += back(d).sum((0, 1))
    if G == 1:
        outs = [t[0] for t in outs]
    return dict(zip(("dx", "dgamma", "dbeta") if backward else ("y", "mean", "rstd"), outs))


def _exact_norm(case, s):
    norm = torch.linalg.vector_norm(s["g"].double()) * case["scale"]
    return {"norm": norm, "coef": case["scale"] * min(1.0, MAX_NORM / max(norm.item(), 1e-300)) * torch.ones_like(norm), "nonfinite": None}


def _exact_adamw(case, s):
    out, coef = {}, case["scale"]
    if case["clip"]:
        out = _exact_norm(case, s)
        coef = out["coef"].float().item()   # held in fp32
    t = s["t"] + 1
    d = {k: s[k].double() for k in ("p", "g", "decay")}
    at = s.get("at")

    def old(q, scale, top, power):
        """an 8-bit state's values: its codes' share of the top one, to a power"""
        share = (q.double() / top)[at]
        return share.sign() * share.abs().pow(power) * scale.double()[at // BLOCK]

    g = d["g"] * coef
    m = s["m"].double() if at is None else old(s["m"], s["m_scale"], 127.0, 2)
    v = s["v"].double() if at is None else old(s["v"], s["v_scale"], 255.0, 4)
    m, v = B1 * m + (1 - B1) * g, B2 * v + (1 - B2) * g.square()
    step = (m / (1 - B1 ** t)) / (torch.sqrt(v / (1 - B2 ** t)) + ADAM_EPS) + d["decay"] * d["p"]
    p = d["p"] - LR * step
    if at is not None:
        def coded(x, top, root, least):
            x = torch.zeros(s["places"], dtype=torch.float64, device=x.device).index_copy(0, at, x.float().double())
            size = x.abs().view(-1, BLOCK)
            high = size.max(1, keepdim=True).values
            q = torch.round(top * (size / high.clamp(min=1e-300)).pow(root))
            q = torch.where(size > 0, q.clamp(min=least), q)
            return (x.sign().view(-1, BLOCK) * (q / top).pow(1 / root) * high).view(-1)
        m, v = coded(m, 127.0, 0.5, 0.0), coded(v, 255.0, 0.25, 1.0)
    out |= {"m": m, "v": v, "p": p}
    if s["low"] is not None:
        out["low"] = p
    return out


def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"].startswith("gn"):
        return _exact_gn(case, s)
    return _exact_adamw(case, s) if case["kind"] == "adamw" else _exact_norm(case, s)

"""AdamW over many tensors, the norm of their gradients and the values of 8-bit
states, against their definitions in 64 bits.

Everything between the fp32 inputs and results is formed in fp64: m and v are off by
half a unit in the last place (2^-24) and a few fp64 roundings (1e-15 of the terms).
The step takes m and v as they are stored, so the parameter's change u lr is off by
three such half units of m and v (m once, v's root half), rounded up to 2^-22 of it,
where the oracle rounds m or v to the other side.  8-bit codes are equal: what the two
sides form differs by 1e-15, and a code changes at 1 of 1e12 such places."""
import math

import pytest
import torch

from paper_1910_13444_amd import pigan
from paper_1910_13444_amd.train import AdamW
from _layers import DT, check

pytestmark = pytest.mark.gpu

LR, B1, B2, EPS = 1e-2, 0.5, 0.9, 1e-8
COUNTS = [1, 3, 255, 256, 257, 0, 4, 4095, 4096, 4097, 31, 10007, 8192, 2]


def _case(seed, counts, gdt=("fp32",), copy=(None,), gap=1):
    """Parameters and gradients as views, `gap` elements apart, of flat buffers that
    hold 7 in the gaps."""
    gen = torch.Generator().manual_seed(seed)
    sizes, total = counts, sum(counts) + gap * (len(counts) + 1)
    flat = {k: torch.full((total,), 7.0, dtype=DT[k]).cuda() for k in ("fp32", "bf16", "fp16")}
    masters = torch.full((total,), 7.0, dtype=torch.float32).cuda()
    lows = {k: torch.full((total,), 7.0, dtype=DT[k]).cuda() for k in ("bf16", "fp16")}
    ps, gs, cs, at = [], [], [], gap
    for i, n in enumerate(sizes):
        d, c = gdt[i % len(gdt)], copy[i % len(copy)]
        p, g = masters[at:at + n], flat[d][at:at + n]
        p.copy_(torch.randn(n, generator=gen, dtype=torch.float32) * 0.1)
        ps.append(p)
        gs.append(g)
        cs.append(None if c is None else lows[c][at:at + n])
        at += n + gap
    decay = [0.0 if i % 3 == 2 else 0.05 * (i + 1) for i in range(len(sizes))]
    return gen, ps, gs, cs, decay, (masters, flat, lows)


def _fill(gen, gs, spread=3.0):
    for g in gs:
        size = torch.exp(spread * torch.randn(g.shape, generator=gen, dtype=torch.float32))
        g.copy_((torch.randn(g.shape, generator=gen, dtype=torch.float32) * size * 1e-3).clamp(-6e4, 6e4))


def _codes(x, top, root, least):
    """(codes, scale) of a block in 64 bits"""
    s = x.abs().max()
    if s == 0:
        return torch.zeros_like(x), s
    q = (top * (x.abs() / s) ** root).round()
    q = torch.where(x != 0, q.clamp(min=least), q)
    return q * x.sign(), s


class Oracle:
    """The step in 64 bits; 8-bit states as the values their codes stand for."""

    def __init__(self, ps, bits):
        self.p = [p.double().cpu() for p in ps]
        self.m = [torch.zeros_like(p) for p in self.p]
        self.v = [torch.zeros_like(p) for p in self.p]
        self.bits = bits

    def step(self, gs, t, decay, scale, lr=LR):
        """per tensor: (p, error, m, v, their errors, codes and scales)"""
        out = []
        for i, g in enumerate(gs):
            g = g.double().cpu() * scale
            m, v = B1 * self.m[i] + (1 - B1) * g, B2 * self.v[i] + (1 - B2) * g * g
            e_m = 4e-16 * (B1 * self.m[i].abs() + (1 - B1) * g.abs())
            ms, vs = m.float().double(), v.float().double()
            u = ms / (1 - B1 ** t) / ((vs / (1 - B2 ** t)).sqrt() + EPS)
            p = self.p[i] - lr * (u + decay[i] * self.p[i])
            e_p = 2.0 ** -22 * lr * u.abs() + 4e-16 * (self.p[i].abs() + lr * u.abs())
            codes = None
            if self.bits == 8:
                codes, mv, vv = [], [], []
                for k in range(0, len(g), 256):
                    qm, sm = _codes(ms[k:k + 256], 127.0, 0.5, 0.0)
                    qv, sv = _codes(vs[k:k + 256], 255.0, 0.25, 1.0)
                    codes.append((qm, sm, qv, sv))
                    mv.append(qm * qm.abs() * (sm / 127.0 ** 2))
                    vv.append(qv ** 4 * (sv / 255.0 ** 4))
                cat = lambda parts: torch.cat(parts) if parts else torch.zeros(0, dtype=torch.float64)   # noqa: E731
                m, v = cat(mv), cat(vv)
            out.append((p, e_p, m, v, e_m, codes))
            self.m[i], self.v[i], self.p[i] = m, v, p
        return out


def _check_step(opt, ps, cs, oracle, want):
    bits = oracle.bits
    values = opt.states()
    for i, (p, e_p, m, v, e_m, codes) in enumerate(want):
        check(ps[i], p, e_p, "fp32", f"p{i}")
        if cs[i] is not None:
            assert torch.equal(cs[i], ps[i].to(cs[i].dtype)), i
        at, n = opt.starts[i], len(p)
        if bits == 32:
            check(opt.m[at:at + n], m, e_m, "fp32", f"m{i}")
            check(opt.v[at:at + n], v, 4e-16 * v, "fp32", f"v{i}")
        else:
            for k, (qm, sm, qv, sv) in enumerate(codes):
                a, b = at + 256 * k, (at + 256 * k) // 256
                assert torch.equal(opt.m[a:a + len(qm)].cpu().double(), qm), (i, k)
                assert torch.equal(opt.v[a:a + len(qv)].cpu().double(), qv), (i, k)
                assert opt.m_scale[b].item() == sm and opt.v_scale[b].item() == sv, (i, k)
            check(values[0][at:at + n], m, 4e-16 * m.abs(), "fp32", f"value of m{i}")
            check(values[1][at:at + n], v, 4e-16 * v, "fp32", f"value of v{i}")
        # the next step begins at what is stored
        oracle.p[i] = ps[i].double().cpu()
        if bits == 32:
            oracle.m[i], oracle.v[i] = (t[at:at + n].double().cpu() for t in (opt.m, opt.v))


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("gdt", [("fp32",), ("bf16", "fp16", "fp32")])
def test_steps(bits, gdt):
    gen, ps, gs, cs, decay, (masters, _, lows) = _case(bits, COUNTS, gdt, (None, "bf16", "fp16"))
    opt = AdamW(ps, gs, LR, B1, B2, EPS, decay, bits, cs)
    oracle = Oracle(ps, bits)
    for t in range(1, 5):
        _fill(gen, gs)
        opt.step(0.5)
        _check_step(opt, ps, cs, oracle, oracle.step(gs, t, decay, 0.5))
    # what lies between the tensors, and behind the last one, is as it was
    for buf, views in ((masters, ps), *((lows[k], [c for c in cs if c is not None and c.dtype == DT[k]]) for k in lows)):
        for view in views:
            view.fill_(7.0)
        assert torch.equal(buf, torch.full_like(buf, 7.0))
    if bits == 8:   # the pads of a tensor's last block
        for i, p in enumerate(ps):
            end = opt.starts[i] + p.numel()
            pad = -(-p.numel() // 256) * 256 + opt.starts[i]
            assert not opt.m[end:pad].any() and not opt.v[end:pad].any()


def test_clipped_steps():
    """The factor of grad_norm, read on the device."""
    for bits in (32, 8):
        gen, ps, gs, cs, decay, _ = _case(2, COUNTS, ("fp32", "bf16"), gap=3)
        opt = AdamW(ps, gs, LR, B1, B2, EPS, decay, bits)
        oracle = Oracle(ps, bits)
        for t, most in ((1, 1e-3), (2, 1e9)):
            _fill(gen, gs)
            norm, coef, flag = opt.grad_norm(most, 0.25)
            want = 0.25 * torch.cat([g.double().cpu() for g in gs]).norm()
            check(norm, want, 1e-14 * want, "fp32", "norm")
            check(coef, 0.25 * (most / want if want > most else torch.ones_like(want)), torch.tensor(1e-15, dtype=torch.float64), "fp32", "coef")
            assert flag.item() == 0 and norm.shape == coef.shape == flag.shape == ()
            opt.step(coef, flag)
            _check_step(opt, ps, cs, oracle, oracle.step(gs, t, decay, coef.item()))


@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
def test_norms(dtype):
    gen = torch.Generator().manual_seed(3)
    for sizes in ([1], [0, 1, 0], [4096], [5, 4095, 4097, 9], [7] * 2500, [3_000_001]):
        flat = (torch.randn(sum(sizes) + 1, generator=gen, dtype=torch.float32) * 3).to(DT[dtype]).cuda()
        grads = list(flat[1:].split(sizes))
        table = pigan.TensorTable(grads)
        want = torch.cat(grads).double().cpu().norm()
        for max_norm, scale in ((float("inf"), 1.0), (0.5, 0.125), (want.item() * 2, 1.0)):
            norm, coef, flag = pigan.grad_norm(table, max_norm, scale)
            w = scale * want
            check(norm, w, 1e-13 * w, "fp32", "norm")
            check(coef, torch.tensor(scale * min(1.0, max_norm / w.item()), dtype=torch.float64), torch.tensor(1e-13), "fp32", "coef")
            assert flag.item() == 0
        again = pigan.grad_norm(table, 0.5)
        assert all(torch.equal(a, b) for a, b in zip(again, pigan.grad_norm(table, 0.5)))
        for bad in (float("nan"), float("inf"), -float("inf")):
            keep = flat[-1].item()
            flat[-1] = bad
            norm, coef, flag = pigan.grad_norm(table, 0.5)
            assert flag.item() == 1 and not math.isfinite(norm.item())
            flat[-1] = keep
        flat.zero_()
        norm, coef, flag = pigan.grad_norm(table, 0.5, 0.25)
        assert norm.item() == 0 and coef.item() == 0.25 and flag.item() == 0


def test_sizes_beyond_fp32_squares():
    """Gradients whose squares fp32 does not hold."""
    for v in (3e38, 1e-38, 1e-44):
        g = torch.full((1000,), v, dtype=torch.float32).cuda()
        norm, coef, flag = pigan.grad_norm(pigan.TensorTable([g]), 1e-30)
        want = g.double().cpu().norm()
        assert flag.item() == 0
        check(coef, (1e-30 / want).clamp(max=1), torch.tensor(1e-60, dtype=torch.float64), "fp32", "coef")
        check(norm, want, 1e-13 * want, "fp32", "norm") if want < 3e38 else None


def test_a_skipped_step_changes_nothing():
    for bits in (32, 8):
        gen, ps, gs, cs, decay, bufs = _case(4, COUNTS, copy=("bf16",))
        opt = AdamW(ps, gs, LR, weight_decay=decay, state_bits=bits, copies=cs, capturable=bits == 8)
        _fill(gen, gs)
        opt.step()
        held = [t.clone() for t in (bufs[0], bufs[2]["bf16"], *opt.states(), opt.m, opt.v)]
        skip = torch.ones((1,), dtype=torch.int32, device="cuda")
        opt.step(1.0, skip, count=False)
        now = (bufs[0], bufs[2]["bf16"], *opt.states(), opt.m, opt.v)
        assert all(torch.equal(a, b) for a, b in zip(held, now))
        assert opt.count is None or opt.count.item() == 1
        skip.zero_()
        opt.step(1.0, skip)
        assert not torch.equal(bufs[0], held[0])


def test_zero_gradients_and_range_of_the_codes():
    p = torch.ones(600, dtype=torch.float32, device="cuda")
    g = torch.zeros(600, dtype=torch.float32, device="cuda")
    opt = AdamW([p], [g], LR, B1, B2, EPS, 0.1, state_bits=8)
    opt.step()
    assert torch.equal(p, torch.full_like(p, 1 - LR * 0.1))
    assert not opt.m.any() and not opt.v.any() and not opt.m_scale.any()
    # Twelve decades in a block, then no gradient.  A code stands for at most four times m
    # (half a code, squared, is taken for one) and at least (1 / 1.5)^4 of v.  So in the
    # second step m <= B1 4 (0.5 g) = g, over 1 - B1^2, and v >= B2 0.197 (0.1 g^2), over
    # 1 - B2^2: a step of at most 1.34 / 0.305 lr, where a v of 0 would give m / eps.
    g.copy_(torch.logspace(-12, 0, 600, dtype=torch.float32))
    p.zero_()
    opt = AdamW([p], [g], LR, B1, B2, EPS, state_bits=8)
    opt.step()
    assert (opt.v[:600] > 0).all()
    before = p.clone()
    g.zero_()
    opt.step()
    assert ((p - before).abs() <= 4.4 * LR).all()


def test_halfway_codes_are_even():
    """m = s / 4 lies halfway between the codes 63 and 64, v = s / 16 between 127 and 128."""
    n = 4000
    gen = torch.Generator().manual_seed(9)
    tops = torch.randn(n, generator=gen, dtype=torch.float32) * torch.exp2(torch.randint(-20, 4, (n,), generator=gen).to(torch.float32))
    g = (tops[:, None] * torch.full((256,), 2.0 ** -6, dtype=torch.float32)).contiguous()
    g[:, 0], g[:, 1], g[:, 200] = tops, tops / 4, -tops / 4
    g = g.view(-1).cuda()
    opt = AdamW([torch.zeros_like(g)], [g], LR, B1, B2, EPS, state_bits=8)
    opt.step()
    m, v = (t.view(n, 256).cpu().int() for t in (opt.m, opt.v))
    sign = tops.sign().int()
    assert torch.equal(m[:, 0], 127 * sign) and torch.equal(m[:, 1], 64 * sign) and torch.equal(m[:, 200], -64 * sign)
    assert (v[:, 0] == 255).all() and (v[:, 1] == 128).all() and (v[:, 200] == 128).all()


def test_gradients_that_are_not_finite():
    for bad in (float("nan"), float("inf"), -float("inf")):
        p = torch.zeros(1024, dtype=torch.float32, device="cuda")
        g = torch.full((1024,), 0.5, dtype=torch.float32, device="cuda")
        want = p.clone()
        opt8, opt32 = (AdamW([t], [g], LR, state_bits=b) for t, b in ((p, 8), (want, 32)))
        g[300] = bad
        opt8.step()
        opt32.step()
        assert torch.isnan(opt8.m_scale[1]) and torch.isnan(opt8.v_scale[1])
        m, v = opt8.states()
        assert torch.isnan(m[256:512]).all() and torch.isnan(v[256:512]).all()
        rest = torch.arange(1024, device="cuda").div(256, rounding_mode="floor") != 1
        assert torch.isfinite(m[rest]).all() and torch.isfinite(p[rest]).all()
        others = torch.arange(1024, device="cuda") != 300
        assert torch.equal(p[others], want[others]) and torch.isfinite(want[others]).all()
        assert torch.isfinite(opt32.m[others]).all() and not math.isfinite(opt32.m[300].item())


@pytest.mark.parametrize("bits", [32, 8])
def test_captured_steps_count_their_replays(bits):
    """A captured clipped step, replayed with new gradients and eager work between,
    against eager steps; one replay is skipped by its flag."""
    gen, ps, gs, cs, decay, _ = _case(5, COUNTS, copy=("fp16",))
    eager = [p.clone() for p in ps]
    make = dict(weight_decay=decay, state_bits=bits)
    a = AdamW(ps, gs, LR, copies=cs, capturable=True, **make)
    b = AdamW(eager, gs, LR, **make)
    _fill(gen, gs)

    def one():
        norm, coef, flag = a.grad_norm(0.01)
        a.step(coef, flag)

    graph = pigan.StepGraph(one)   # runs it once
    norm, coef, flag = b.grad_norm(0.01)
    b.step(coef, flag)
    for k in range(5):
        _fill(gen, gs)
        if k == 2:
            gs[3][1] = float("nan")
        graph.replay()
        torch.cuda.synchronize()
        norm, coef, flag = b.grad_norm(0.01)
        b.step(coef, flag, count=k != 2)
        assert all(torch.equal(x, y) for x, y in zip(ps, eager)), k
        assert torch.equal(a.m, b.m) and torch.equal(a.v, b.v) and a.count.item() == b.t
        assert all(torch.equal(c, p.half()) for c, p in zip(cs, ps))


@pytest.mark.parametrize("bits", [32, 8])
def test_steps_beyond_the_caches(bits):
    """A step that moves more than 192 MiB gives the bits of the same step in parts."""
    gen = torch.Generator(device="cuda").manual_seed(7)
    parts, n = 8, 256 * 8001
    ps, gs, cs = [], [], []
    for _ in range(2):
        ps.append(torch.empty(parts * n, dtype=torch.float32, device="cuda").normal_(0.0, 0.1, generator=gen.manual_seed(7)))
        cs.append(torch.empty(parts * n, dtype=torch.bfloat16, device="cuda"))
    g = torch.empty(parts * n, dtype=torch.float32, device="cuda")
    whole = AdamW([ps[0]], [g], LR, B1, B2, EPS, 0.01, bits, [cs[0]])
    split = [AdamW([p], [q], LR, B1, B2, EPS, 0.01, bits, [c]) for p, q, c in zip(ps[1].split(n), g.split(n), cs[1].split(n))]
    for _ in range(2):
        g.normal_(0.0, 1e-3, generator=gen)
        whole.step()
        for opt in split:
            opt.step()
        assert torch.equal(ps[0], ps[1]) and torch.equal(cs[0], cs[1])
        for k in range(2):
            assert torch.equal(whole.states()[k], torch.cat([opt.states()[k] for opt in split]))


def test_another_stream():
    gen, ps, gs, cs, decay, _ = _case(6, [100000, 77])
    other = [p.clone() for p in ps]
    a, b = AdamW(ps, gs, LR), AdamW(other, gs, LR)
    _fill(gen, gs)
    a.step(a.grad_norm(0.1)[1])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        b.step(b.grad_norm(0.1)[1])
    side.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(ps, other))


def test_refusals():
    p, g = (torch.zeros(8, dtype=torch.float32, device="cuda") for _ in range(2))
    for bad in (dict(params=[p], grads=[]), dict(params=[p], grads=[g, g]), dict(params=[p.half()], grads=[g]),
                dict(params=[p], grads=[g.double()]), dict(params=[p], grads=[g[:4]]), dict(params=[p[::2]], grads=[g[:4]]),
                dict(params=[p], grads=[g.cpu()]), dict(params=[p], grads=[g], copies=[p]), dict(params=[], grads=[]),
                dict(params=[p], grads=[g], copies=[p[:4].half()]), dict(params=[p], grads=[g], weight_decay=[0.0, 0.1]),
                dict(params=[p], grads=[g], state_bits=16)):
        with pytest.raises(ValueError):
            AdamW(lr=LR, **bad)
    for bad in (dict(params=[p, p], grads=[g, g]), dict(params=[p], grads=[p]), dict(params=[p[:5], p[4:]], grads=[g[:5], g[4:]]),
                dict(params=[p], grads=[g], weight_decay=-1.0), dict(params=[p], grads=[g], weight_decay=float("nan"))):
        with pytest.raises(pigan.PiganError):
            AdamW(lr=LR, **bad)
    AdamW([p[:4], p[4:]], [g[:4], g[:4]], LR)   # one gradient of two parameters
    opt = AdamW([p], [g], LR)
    for bad in (dict(scale=0.0), dict(scale=float("nan")), dict(scale=-1.0)):
        with pytest.raises(pigan.PiganError):
            opt.step(**bad)
        with pytest.raises(pigan.PiganError):
            opt.grad_norm(**bad)
    with pytest.raises(pigan.PiganError):
        opt.grad_norm(0.0)
    for bad in (dict(scale=g), dict(scale=g[:1].double()), dict(skip=g[:1]), dict(skip=torch.zeros(1, dtype=torch.int32))):
        with pytest.raises(ValueError):
            opt.step(**bad)
    with pytest.raises(pigan.PiganError):
        pigan.adamw_update(pigan.TensorTable([g]), LR, B1, B2, EPS, 1)
    for bad in (dict(lr=float("inf")), dict(beta1=1.0), dict(beta2=-0.1), dict(eps=-1.0)):
        with pytest.raises(pigan.PiganError):
            AdamW([p], [g], **{"lr": LR, **bad}).step()

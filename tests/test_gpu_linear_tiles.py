"""Every tile and split of the linear layer's products at ragged sizes, and
matrices whose elements stand more than 2^32 apart, against the formulas in 64
bits.

A size stands in a list for the variant that the host's rule takes for it, the
smallest found: sides of 64, 128 and 256, "64K" (four groups of waves share a
contraction), a contraction in parts, both reverse products in one launch.  Most
sides end inside a tile, and the contractions inside a stage of 64 values.
(groups, rows, inputs, outputs); 16-byte rows."""
import pytest
import torch

from paper_1910_13444_amd import pigan
from _layers import EPS32, act64, check, mm64, sum_error, vector
from test_gpu_linear import _backward, _forward, _seed

pytestmark = pytest.mark.gpu

FORWARD16 = [(1, 282, 248, 288), (1, 81, 2576, 96),          # 64, 64 in parts
             (1, 182, 736, 152), (5, 396, 1264, 8),          # 64K
             (1, 1398, 200, 3080), (2, 17704, 208, 72),      # 128
             (1, 644, 8536, 1512), (1, 2078, 1312, 3976)]    # 128 in parts, 256
FORWARD32 = [(1, 740, 384, 352), (1, 314, 664, 488),         # 64, 64 in parts
             (1, 361, 488, 576), (5, 4644, 32, 136),         # 64K, 128
             (1, 976, 2336, 456), (1, 3848, 200, 2120),      # 128 in parts, 256
             (1, 3782, 4376, 400)]                           # 256 in parts
BACKWARD16 = [(1, 1, 8, 8), (1, 1665, 8, 8),                 # both: 64, dw in parts
              (1, 147, 2952, 1352), (1, 4213, 744, 472),     # both: 128, dw in parts
              (1, 1, 8, 2696), (1, 56539, 8, 8),             # dx 64 in parts, dw 64; the reverse
              (1, 485, 8, 3216), (17, 1, 8, 1680),           # dw 64K, dx 64K
              (1, 134, 1032, 3848), (1, 1763, 2800, 232),    # dw 128, dx 128
              (1, 7932, 88, 4992), (1, 1714, 1336, 4936),    # dw 128 in parts, dx 128 in parts
              (17, 187, 3792, 1480)]                         # dx and dw 256
BACKWARD32 = [(1, 1, 8, 8), (1, 321, 8, 8),                  # both: 64, dw in parts
              (17, 2, 600, 208), (1, 16386, 72, 72),         # both: 128, dw in parts
              (1, 333, 8, 848), (1, 29386, 8, 8),            # dw 64 in parts, dx 64
              (1, 453, 224, 896), (1, 71, 2744, 480),        # dw 64K, dx 64K
              (17, 3, 72, 2000), (1, 32860, 72, 8),          # dw 128, dx 128
              (1, 1772, 344, 1224), (1, 513, 944, 1320),     # dw 128 in parts, dx 128 in parts
              (1, 130, 1664, 5000), (17, 179, 3832, 200),    # dw 256, dx 256
              (2, 15395, 400, 392), (1, 147, 8128, 3480)]    # dw 256 in parts, dx 256 in parts


@pytest.mark.parametrize("dtype,size", [("bf16", s) for s in FORWARD16] + [("fp16", s) for s in FORWARD16[::2]] +
                         [("fp32", s) for s in FORWARD32])
def test_forward_variants(dtype, size):
    print(f"linear forward {size} {dtype}", flush=True)
    G, M, K, N = size
    _forward(_seed(*size), G, M, K, N, dtype, "gelu", True, True)
    _forward(_seed(*size), G, M, K, N, dtype, "none", False, False)


@pytest.mark.parametrize("dtype,size", [("bf16", s) for s in BACKWARD16] + [("fp16", s) for s in BACKWARD16[::2]] +
                         [("fp32", s) for s in BACKWARD32])
def test_backward_variants(dtype, size):
    print(f"linear backward {size} {dtype}", flush=True)
    G, M, K, N = size
    _backward(_seed(*size), G, M, K, N, dtype, "silu", True)
    _backward(_seed(*size), G, M, K, N, dtype, "none", False)


@pytest.mark.parametrize("ld", [2 ** 20 + 8, 2 ** 21 + 5])
def test_elements_beyond_32_bits(ld):
    """Rows so far apart that the last ones are more than 2^32 elements from the
    first: with 16-byte rows as the loads of whole pieces take them, and odd."""
    rows, K, N = 2 ** 32 // ld + 70, 72, 136
    gen = _seed(ld)
    buf = torch.empty(rows * ld, dtype=torch.bfloat16, device="cuda")
    print(f"{rows} rows of {ld}: {buf.numel() * 2 / 2 ** 30:.1f} GiB", flush=True)

    def at(col, cols):
        t = buf.as_strided((rows, cols), (ld, 1), col)
        t.copy_(torch.randn((rows, cols), generator=gen, dtype=torch.float32))
        return t

    x, r, g, out, pre, dx = at(0, K), at(1000, N), at(2000, N), at(3000, N), at(4000, N), at(5000, K)
    w = (torch.randn((N, K), generator=gen, dtype=torch.float32) * K ** -0.5).to(torch.bfloat16).cuda()
    b = vector(gen, None, N)
    pigan.linear(x, w, b, "tanh", residual=r, out=out, pre=pre)
    a, rss = mm64(x, w)
    a, err = a + b.double().cpu(), sum_error(K, rss)
    check(pre, a, err + EPS32 * a.abs(), "bf16", "pre")
    check(out, a.tanh() + r.double().cpu(), 1.13 * err + 2e-5, "bf16", "y")
    _, dw, db = pigan.linear_backward(g, x, w, dx=dx)
    want, rss = mm64(g, w.T)
    check(dx, want, sum_error(N, rss), "bf16", "dx")
    want, rss = mm64(g.T, x.T)
    check(dw, want, sum_error(rows, rss), "fp32", "dw")
    g64 = g.double().cpu()
    check(db, g64.sum(0), sum_error(rows, g64.square().sum(0).sqrt()), "fp32", "db")
    pigan.act_backward(g, pre, "tanh", out=out)
    want = g64 * act64(pre.double().cpu(), "tanh")[1]
    check(out, want, 4e-6 * want.abs(), "bf16", "g")
    _, mean, rstd = pigan.layer_norm(r, out=out)
    r64 = r.double().cpu()
    m = r64.mean(1, keepdim=True)
    s = ((r64 - m).square().mean(1, keepdim=True) + 1e-5) ** -0.5
    xh = (r64 - m) * s
    check(out, xh, 1e-5 * (1 + xh.abs()), "bf16", "normalised")
    _, dgamma, dbeta = pigan.layer_norm_backward(g, r, mean, rstd, dx=out)
    want = s * (g64 - g64.mean(1, keepdim=True) - xh * (g64 * xh).mean(1, keepdim=True))
    check(out, want, 1e-5 * (1 + want.abs()), "bf16", "norm's dx")
    check(dgamma, (g64 * xh).sum(0), sum_error(rows, (g64 * xh).square().sum(0).sqrt()) + 1e-5 * rows ** 0.5, "fp32", "dgamma")
    check(dbeta, g64.sum(0), sum_error(rows, g64.square().sum(0).sqrt()), "fp32", "dbeta")

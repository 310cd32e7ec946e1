"""The linear layer's pipelined products on odd sizes and unaligned rows: fp32
planes and 16-bit copies of whole pieces, results whose columns end inside an
eight, in every tile and split, against the formulas in 64 bits.  The sizes are
odd ones beside those that reach each variant with whole pieces; 16-bit sizes are
large enough that the operands are copied, or of one of each side's."""
import pytest

from paper_1910_13444_amd import pigan
from test_gpu_linear import _backward, _forward, _seed

pytestmark = pytest.mark.gpu

FORWARD32 = [(1, 743, 387, 355), (1, 317, 667, 491), (1, 363, 489, 577), (5, 4645, 33, 137), (1, 977, 2337, 457),
             (1, 3849, 201, 2121), (1, 3783, 4377, 401)]
FORWARD16 = [(1, 2079, 1313, 3977), (1, 4001, 2050, 2051), (1, 645, 8537, 1513), (1, 4100, 4099, 1028),
             (16, 515, 1021, 1027), (1, 183, 737, 153)]
BACKWARD32 = [(1, 322, 9, 11), (17, 3, 601, 209), (1, 16387, 73, 75), (1, 335, 11, 849), (1, 455, 225, 897),
              (1, 73, 2745, 481), (1, 1773, 345, 1225), (1, 515, 945, 1321), (1, 131, 1665, 5001), (2, 15397, 401, 393)]
BACKWARD16 = [(1, 149, 2953, 1353), (1, 4215, 745, 473), (1, 7933, 91, 4993), (1, 1715, 1337, 4937), (17, 189, 3793, 1481),
              (1, 2003, 1001, 999), (16, 513, 515, 517), (1, 487, 13, 3217)]


@pytest.mark.parametrize("dtype,size", [("fp32", s) for s in FORWARD32] + [("bf16", s) for s in FORWARD16] +
                         [("fp16", s) for s in FORWARD16[::2]])
def test_forward_odd(dtype, size):
    print(f"linear forward {size} {dtype}", flush=True)
    G, M, K, N = size
    _forward(_seed(*size), G, M, K, N, dtype, "silu", True, True)
    _forward(_seed(*size), G, M, K, N, dtype, "none", False, False, ld=lambda c: c + 3, offset=5)


@pytest.mark.parametrize("dtype,size", [("fp32", s) for s in BACKWARD32] + [("bf16", s) for s in BACKWARD16] +
                         [("fp16", s) for s in BACKWARD16[::2]])
def test_backward_odd(dtype, size):
    print(f"linear backward {size} {dtype}", flush=True)
    G, M, K, N = size
    _backward(_seed(*size), G, M, K, N, dtype, "gelu", True)
    _backward(_seed(*size), G, M, K, N, dtype, "none", False, ld=lambda c: c + 3, offset=5)


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("K,N", [(2000, 1003), (1003, 2000)])
def test_one_operand_is_copied(dtype, K, N):
    """x or g has whole pieces, the other one not; then rows of whole pieces that
    begin at an odd element."""
    _forward(_seed(K), None, 4001, K, N, dtype, "none", True, False)
    _backward(_seed(K), None, 4001, K, N, dtype, "none", False)
    _backward(_seed(K), None, 4001, 1000, 1008, dtype, "tanh", True, ld=lambda c: c + 8, offset=1)


def test_workspace_follows_the_alignment():
    """Whole pieces need no copy; the same sizes one element on do, and the call
    takes what its query says."""
    import torch
    x = torch.zeros((4096, 4104), dtype=torch.bfloat16, device="cuda")
    w = torch.zeros((4096, 4096), dtype=torch.bfloat16, device="cuda")
    for t, need in ((x[:, :4096], False), (x[:, 1:4097], True)):
        used = torch.cuda.memory_allocated()
        torch.cuda.reset_peak_memory_stats()
        y = pigan.linear(t, w)
        torch.cuda.synchronize()
        extra = torch.cuda.max_memory_allocated() - used - y.numel() * 2
        assert (extra >= 4096 * 4096 * 2) == need
        del y

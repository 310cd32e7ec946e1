"""The linear layer's forward pass on 9 to 64 rows of wide layers: strips of 16
rows or tiles, by the modelled time, in parts as well."""
import pytest

from test_gpu_linear import _forward, _seed

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("G,M,K,N", [(None, 9, 1000, 2056), (None, 16, 1024, 8193), (None, 33, 1024, 8192), (None, 64, 1024, 8200),
                                     (None, 64, 8192, 2048), (None, 61, 8193, 2047), (4, 64, 1032, 2040), (8, 17, 1500, 1501)])
def test_few_rows_of_wide_layers(dtype, G, M, K, N):
    print(f"linear forward {G} x {M} x {K} x {N} {dtype}", flush=True)
    _forward(_seed(M, K, N), G, M, K, N, dtype, "gelu", True, True)
    _forward(_seed(M, K, N), G, M, K, N, dtype, "none", False, False, ld=lambda c: c + 3, offset=1)

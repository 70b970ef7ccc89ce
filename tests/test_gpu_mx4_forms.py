"""Few tokens through wide layers: the two entry points of a product with few rows take one form."""
import pytest
import torch

from paper_2411_10948_gb300 import microscale as X
from paper_2411_10948_gb300 import native as N

pytestmark = pytest.mark.gpu


def tensor(rows, cols, dtype, seed):
    """Channels of widely different size, so that the order of a sum shows."""
    g = torch.Generator("cuda").manual_seed(seed)
    x = torch.randn((rows, cols), generator=g, device="cuda")
    return x.mul_(torch.randn(cols, generator=g, device="cuda").mul_(5).exp_()).to(dtype)


# 9473 columns of output are the first that make 38 tiles of 256, a quarter of 152 SMs
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("M", [1, 5, 17, 32])
@pytest.mark.parametrize("K,Nn", [(2304, 9472), (2304, 9473), (4096, 11008), (700, 20001)])
def test_linear_is_the_quantizer_and_the_product_at_any_width(M, K, Nn, dtype):
    x = tensor(M, K, dtype, M + K)
    w = X.Mx4Tensor.alloc(K, Nn, "cuda", rows=False).quantize(tensor(K, Nn, dtype, 3))
    xq = X.Mx4Tensor.alloc(M, K, "cuda", cols=False).quantize(x)
    y, want = torch.zeros((M, Nn), dtype=dtype, device="cuda"), torch.zeros((M, Nn), dtype=dtype, device="cuda")
    N.shiftquant_mx4_linear(x, w.codes_t, w.scales_t, y, None, None, w.status)
    N.shiftquant_mx4_gemm(xq.codes, xq.scales, w.codes_t, w.scales_t, K, want, w.status)
    assert torch.equal(y, want) and w.status.item() == 0

"""The residual stream of a norm in place: sum over the residual, dx over its gradient (GPU)."""
import pytest
import torch

from paper_2411_10948_gb300 import microscale as X

pytestmark = pytest.mark.gpu
TYPES = [torch.float32, torch.bfloat16, torch.float16]


def tensor(rows, cols, dtype, seed):
    return torch.randn((rows, cols), generator=torch.Generator("cuda").manual_seed(seed), device="cuda").to(dtype)


# a warp's row, several warps', two to four chunks a thread, aligned or not, and rows that are swept
# three times; more rows than blocks of one wave
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("layer", [False, True])
@pytest.mark.parametrize("M,C", [(5, 48), (5, 61), (3000, 521), (700, 1155), (400, 8200), (330, 11007), (400, 12300),
                                 (5, 16411), (200, 20000)])
def test_the_residual_stream_in_place(M, C, layer, dtype):
    kind = "layer" if layer else "rms"
    apart, within = X.Norm8(M, C, dtype, kind, "cuda", residual=True), X.Norm8(M, C, dtype, kind, "cuda", residual=True)
    x, res, dy, dsum = (tensor(M, C, dtype, k) for k in range(4))
    gamma, beta = 1 + 0.1 * tensor(1, C, torch.float32, 4)[0], tensor(1, C, torch.float32, 5)[0] if layer else None
    y, total = apart.forward(x, gamma, beta, res)
    within.sum.copy_(res)
    y2, total2 = within.forward(x, gamma, beta, within.sum)
    assert torch.equal(total2, total) and torch.equal(y2, y)
    assert torch.equal(within.codes, apart.codes) and torch.equal(within.scales, apart.scales)
    assert torch.equal(within.stats, apart.stats)
    grads = apart.backward(dy, gamma, dsum)
    within.dx.copy_(dsum)
    for a, b in zip(grads, within.backward(dy, gamma, within.dx)):
        assert (a is None and b is None) or torch.equal(a, b)

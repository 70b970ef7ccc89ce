"""Activations whose input is kept in 8 bits, at inputs far out in both tails (GPU): the definitions
are 0, 1 or the input there."""
import pytest
import torch

from paper_2411_10948_gb300 import microscale as X

pytestmark = pytest.mark.gpu
TYPES = [torch.float32, torch.bfloat16, torch.float16]
ACTS = ["gelu", "gelu_tanh", "silu"]


def magnitudes(dtype):
    # far into both tails of every activation; x^2 leaves FP32 from 1.8e19 on
    top = torch.finfo(dtype).max
    return [m for m in (1e4, 1e10, 1.5e19, 2e19, 1e30, top / 4) if m < top]


def rows_of(values, F, dtype):
    """A row per value: all of its blocks hold that value alone."""
    return torch.tensor(values, dtype=torch.float64).to(dtype).cuda()[:, None].expand(-1, F).contiguous()


# F: 16-byte aligned rows, and rows that are not
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("F", [64, 61])
@pytest.mark.parametrize("act", ACTS)
def test_large_inputs_of_either_sign(act, F, dtype):
    m = magnitudes(dtype)
    h = rows_of(m + [-v for v in m], F, dtype)
    op = X.Act8(h.shape[0], F, dtype, act, False, "cuda")
    y = op.forward(h)
    dy = torch.full_like(h, 0.75)
    dh = op.backward(dy)
    assert op.status.item() == 0
    # the distribution and the logistic function are 1 or below 2^-1000 there: x and 1, or zeros
    assert torch.equal(y, torch.where(h > 0, h, torch.zeros_like(h)))
    assert torch.equal(dh, torch.where(h > 0, dy, torch.zeros_like(h)))

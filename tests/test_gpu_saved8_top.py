"""The largest values of each type kept in 8 bits, on the GPU against 64-bit definitions."""
import pytest
import torch

import microscale_reference as R
from paper_2411_10948_gb300 import microscale as X

pytestmark = pytest.mark.gpu
TYPES = [torch.float32, torch.bfloat16, torch.float16]
ACTS = ["gelu", "gelu_tanh", "silu"]


def kept(x):
    return torch.from_numpy(R.int8(x.double().cpu().numpy())).cuda()


# The largest values of a type keep as 64 2^e, which is 2^128 where the type has FP32's range: what
# stands for them is FP32's largest number, 2^-24 of itself below.
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("F", [64, 61])
@pytest.mark.parametrize("act", ACTS)
def test_the_types_largest_value(act, F, dtype):
    top = torch.finfo(dtype).max
    h = torch.zeros((4, 2 * F), dtype=dtype, device="cuda")
    h[0, :F], h[1, :F], h[0:2, F:] = top, -top, 0.5       # a large, u = 1/2, which 8 bits hold
    h[2:, :F], h[2, F:], h[3, F:] = 2.0, top, -top         # a = 2, which they hold, u large
    op = X.Act8(4, F, dtype, act, True, "cuda")
    y = op.forward(h)
    g = 2.0 ** (-4 if dtype == torch.float16 else -60)     # products stay within the type
    dy = torch.full((4, F), g, dtype=dtype, device="cuda")
    dh = op.backward(dy).double()
    assert op.status.item() == 0
    at, ut = kept(h[:, :F]), kept(h[:, F:])
    assert torch.equal(y[0], h[0, :F] * 0.5) and (y[1] == 0).all()
    # da = dy u~ f'(a~): 1/2 and 0
    assert (dh[0, :F] == g / 2).all() and (dh[1, :F] == 0).all()
    # du = dy f(a~) = dy a~ and 0; the type's rounding of a value 2^-24 below leaves half a unit
    unit = {torch.float32: 2.0 ** -23, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}[dtype]
    assert ((dh[0, F:] - g * at[0]).abs() <= unit * (g * at[0]).abs()).all() and (dh[1, F:] == 0).all()
    # u~ large: dy u~ f'(2), some thirty FP32 operations and units of 2^-22 of terms that sum to 2
    a = torch.full((1, F), 2.0, dtype=torch.float64, device="cuda").requires_grad_()
    if act == "silu":
        f = a * torch.sigmoid(a)
    else:
        f = torch.nn.functional.gelu(a, approximate="tanh" if act == "gelu_tanh" else "none")
    df = torch.autograd.grad(f.sum(), a)[0]
    want = g * ut[2:] * df
    assert ((dh[2:, :F] - want).abs() <= (2.0 ** -16 + unit) * want.abs()).all()


@pytest.mark.parametrize("C", [64, 61, 1031])
def test_norm_of_a_row_whose_squares_overflow(C):
    # 1 / deviation is 0 in FP32: y and dx are 0, not NaN
    x = torch.full((2, C), torch.finfo(torch.float32).max, device="cuda")
    x[1] = 1.0
    op = X.Norm8(2, C, torch.float32, "rms", "cuda")
    gamma = torch.ones(C, device="cuda")
    y, _ = op.forward(x, gamma)
    dx, dgamma, _ = op.backward(torch.full((2, C), 0.5, device="cuda"), gamma)
    assert op.status.item() == 0
    assert (y[0] == 0).all() and (dx[0] == 0).all() and torch.isfinite(dgamma).all()

"""GELU of 16-bit tensors in its lower tail, on the GPU against the 64-bit definition."""
import math

import pytest
import torch

import microscale_reference as R
from paper_2411_10948_gb300 import microscale as X

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
TINY = 2.0 ** -125


def between(got, want, off):
    low, high = (want - off).to(got.dtype).double(), (want + off).to(got.dtype).double()
    bad = ~((low <= got.double()) & (got.double() <= high))
    assert not bad.any(), (int(bad.sum()), (got.double() / want - 1)[bad][:4])


# The lower tail of GELU is small, but 16-bit types hold it to all of their bits: a bound relative to
# the value.  The tail's factor is fitted to 1.3e-5 of itself; the exponent -x^2 / 2 carries two roundings
# and its unit 2 + 1.2 |x^2 / 2| units, which the exponential makes relative; the rest is some
# sixteen operations.
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("F", [512, 511])
def test_gelu_lower_tail(F, dtype):
    low = -12.5 if dtype == torch.bfloat16 else -6.0
    x = torch.linspace(low, -1.0, 4 * F, dtype=torch.float64).reshape(4, F).to(dtype).cuda()
    op = X.Act8(4, F, dtype, "gelu", False, "cuda")
    y = op.forward(x)
    dy = torch.full_like(x, 1024.0)
    dh = op.backward(dy)
    assert op.status.item() == 0
    rel = lambda v: 1.3e-5 + U * (32 + 3.2 * v * v)
    v = x.double()
    cdf = torch.special.erfc(-v / math.sqrt(2)) / 2
    between(y, v * cdf, (v * cdf).abs() * rel(v) + TINY * v.abs())
    v = torch.from_numpy(R.int8(v.cpu().numpy())).cuda()
    cdf, pdf = torch.special.erfc(-v / math.sqrt(2)) / 2, torch.exp(-v * v / 2) / math.sqrt(2 * math.pi)
    want = cdf + v * pdf
    between(dh, 1024 * want, 1024 * (cdf * rel(v) + (v * pdf).abs() * U * (16 + 3.2 * v * v) + U * want.abs() + TINY))

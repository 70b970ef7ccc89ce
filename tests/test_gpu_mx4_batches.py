"""Training layers and MLP blocks on batches of fewer rows than they were made for (GPU): what an
object made for those rows gives, bit for bit."""
import pytest
import torch

from paper_2411_10948_gb300 import microscale as X

pytestmark = pytest.mark.gpu


def tensor(rows, cols, seed, scale=1.0):
    g = torch.Generator("cuda").manual_seed(seed)
    return (torch.randn((rows, cols), generator=g, device="cuda") * scale).to(torch.bfloat16)


# rows that end inside a block of 32, a scale tile of 128 rows or 256 elements of K, and none
@pytest.mark.parametrize("rows", [300, 256, 129, 70, 32, 1, 0])
def test_a_layer(rows):
    M, K, Nn = 300, 200, 136
    lay, own = X.Mx4Linear(M, K, Nn, torch.bfloat16, "cuda"), X.Mx4Linear(rows, K, Nn, torch.bfloat16, "cuda")
    w, x, dy = tensor(K, Nn, 1), tensor(M, K, 2), tensor(M, Nn, 3)
    lay.set_weight(w)
    own.set_weight(w)
    lay.forward(x)                      # a whole batch before it leaves its codes
    lay.backward(dy, seed=5)
    y, (dx, dw) = lay.forward(x[:rows]), lay.backward(dy[:rows], seed=7)
    want, (want_dx, want_dw) = own.forward(x[:rows]), own.backward(dy[:rows], seed=7)
    assert y.shape == (rows, Nn) and torch.equal(y, want)
    assert dx.shape == (rows, K) and torch.equal(dx, want_dx) and torch.equal(dw, want_dw)
    assert lay.status.item() == 0 and own.status.item() == 0
    with pytest.raises(ValueError):
        lay.forward(tensor(M + 1, K, 2))
    with pytest.raises(ValueError):
        lay.backward(tensor(rows + 1, Nn, 3), seed=7)


@pytest.mark.parametrize("rows", [130, 33])
def test_a_block(rows):
    M, C, F = 130, 96, 160
    block, own = X.Mx4MlpBlock(M, C, F, torch.bfloat16, "cuda"), X.Mx4MlpBlock(rows, C, F, torch.bfloat16, "cuda")
    gamma, w1, w2 = torch.ones(C, device="cuda"), tensor(C, 2 * F, 1, 0.1), tensor(F, C, 2, 0.1)
    delta, x, dout, dxn = (tensor(M, C, k) for k in range(3, 7))
    for b in (block, own):
        b.set_weights(gamma, w1, w2)
    block.forward(delta, x)
    block.backward(dout, dxn, seed=3)
    got = block.forward(delta[:rows], x[:rows])
    want = own.forward(delta[:rows], x[:rows])
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    assert torch.equal(block.backward(dout[:rows], dxn[:rows], seed=9), own.backward(dout[:rows], dxn[:rows], seed=9))
    assert torch.equal(block.dw1, own.dw1) and torch.equal(block.dw2, own.dw2)
    assert torch.equal(block.dgamma, own.dgamma) and block.status() == 0

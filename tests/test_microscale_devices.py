"""Objects refuse tensors of another device than their own: the library's calls take addresses, and
one of another device would be read where it is not (no GPU needed)."""
import pytest
import torch

from paper_2411_10948_gb300 import build, microscale as X

F32 = torch.float32


@pytest.fixture(scope="module", autouse=True)
def library():
    build.build_library()


def here(*shape):
    return torch.zeros(shape)


def there(*shape):
    return torch.zeros(shape, device="meta")


def test_tensors_and_layers():
    q = X.Mx4Tensor.alloc(4, 32, "cpu")
    lay = X.Mx4Linear(4, 32, 8, F32, "cpu")
    serve = X.Mx4Linear(4, 32, 8, F32, "cpu", train=False)
    for call in (lambda: q.quantize(there(4, 32)), lambda: q.values(there(4, 32)), lambda: q.values_t(there(32, 4)),
                 lambda: lay.set_weight(there(32, 8)), lambda: lay.forward(there(4, 32)),
                 lambda: serve.forward(there(2, 32)), lambda: lay.backward(there(4, 8), 1)):
        with pytest.raises(ValueError, match="expected, not on meta"):
            call()


def test_activations_and_norms():
    act = X.Act8(4, 32, F32, "silu", False, "cpu")
    norm = X.Norm8(4, 32, F32, "layer", "cpu", residual=True)
    x, p = here(4, 32), here(32)
    for call in (lambda: act.forward(there(4, 32)), lambda: act.backward(there(4, 32)),
                 lambda: norm.forward(there(4, 32), p, p, x), lambda: norm.forward(x, p, p, there(4, 32)),
                 lambda: norm.forward(x, there(32), p, x), lambda: norm.forward(x, p, there(32), x),
                 lambda: norm.backward(there(4, 32), p), lambda: norm.backward(x, p, there(4, 32))):
        with pytest.raises(ValueError, match="expected, not on meta"):
            call()


def test_gamma_of_a_backward_pass():
    norm = X.Norm8(4, 32, F32, "rms", "cpu")
    norm._rows = 4              # as after a forward pass, which needs a GPU
    with pytest.raises(ValueError, match="expected, not on meta"):
        norm.backward(here(4, 32), there(32))

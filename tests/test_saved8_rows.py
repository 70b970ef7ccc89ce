"""A backward pass takes the rows that the last forward pass kept, and refuses others."""
import pytest
import torch

from paper_2411_10948_gb300 import build, microscale as X


@pytest.fixture(scope="module", autouse=True)
def library():
    build.build_library()


def objects(device, train=True):
    """(object, its forward's further arguments, its backward's) of 8 rows x 64 columns."""
    f32, ones = torch.float32, torch.ones(64, device=device)
    lay = X.Mx4Linear(8, 64, 64, f32, device, train=train)
    if device == "cuda":
        lay.set_weight(torch.eye(64, device=device))
    return [(X.Act8(8, 64, f32, "silu", False, device, train=train), (), ()),
            (X.Norm8(8, 64, f32, "rms", device, train=train), (ones,), (ones,)),
            (X.Norm8(8, 64, f32, "layer", device, train=train), (ones, ones), (ones,)),
            (lay, (), (1,))]


@pytest.mark.parametrize("train", [True, False])
@pytest.mark.parametrize("which", range(4))
def test_nothing_kept_is_refused(which, train):
    op, _, args = objects("cpu", train)[which]
    with pytest.raises(ValueError):
        op.backward(torch.zeros(8, 64), *args)


@pytest.mark.gpu
@pytest.mark.parametrize("which", range(3))
def test_rows_of_an_older_call_are_refused(which):
    op, forward, backward = objects("cuda")[which]
    x = torch.randn(8, 64, device="cuda")
    op.forward(x, *forward)
    whole = op.backward(x, *backward)
    first = [t.clone() for t in (whole if isinstance(whole, tuple) else (whole,)) if t is not None]
    op.forward(x[:5], *forward)
    for rows in (8, 4):
        with pytest.raises(ValueError):
            op.backward(x[:rows], *backward)
    op.backward(x[:5], *backward)
    op.forward(x, *forward)
    for _ in range(2):      # what is kept stays until the next forward pass
        again = op.backward(x, *backward)
        again = [t for t in (again if isinstance(again, tuple) else (again,)) if t is not None]
        assert all(torch.equal(a, b) for a, b in zip(first, again))


@pytest.mark.gpu
@pytest.mark.parametrize("which", range(4))
def test_serving_keeps_nothing(which):
    op, forward, backward = objects("cuda", train=False)[which]
    op.forward(torch.randn(8, 64, device="cuda"), *forward)
    with pytest.raises(ValueError):
        op.backward(torch.zeros(8, 64, device="cuda"), *backward)

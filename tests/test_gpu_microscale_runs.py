"""The microscaled objects as programs run them (GPU): a step captured once and replayed, two
blocks on two streams at once, and layers wide enough for the product's CTA pairs."""
import pytest
import torch

import microscale_reference as R
from paper_2411_10948_gb300 import layer as L
from paper_2411_10948_gb300 import microscale as X

pytestmark = pytest.mark.gpu
BF16 = torch.bfloat16


def tensor(rows, cols, seed, scale=1.0, dtype=BF16):
    g = torch.Generator("cuda").manual_seed(seed)
    return (torch.randn((rows, cols), generator=g, device="cuda") * scale).to(dtype)


def block_of(M, C, F, seed):
    b = X.Mx4MlpBlock(M, C, F, BF16, "cuda")
    b.set_weights(1 + 0.1 * tensor(1, C, seed, dtype=torch.float32)[0], tensor(C, 2 * F, seed + 1, 0.1),
                  tensor(F, C, seed + 2, 0.1))
    return b


def outputs(block, delta, x, dout, dxn):
    out, x_new = block.forward(delta, x)
    dx = block.backward(dout, dxn, seed=4)
    return out, x_new, dx, block.dw1, block.dw2, block.dgamma


def test_a_captured_step_replays():
    M, C, F = 200, 256, 352
    block, eager = block_of(M, C, F, 1), block_of(M, C, F, 1)
    args = [tensor(M, C, 10 + k) for k in range(4)]
    got = []
    step = L.CapturedStep(lambda: got.append(outputs(block, *args)))
    for new in (20, 30):                 # other inputs than the captured ones, in their place
        for k, a in enumerate(args):
            a.copy_(tensor(M, C, new + k))
        step.replay()
        for a, b in zip(got[-1], outputs(eager, *args)):
            assert torch.equal(a, b)
    assert block.status() == 0


def test_a_captured_layer_of_few_tokens_replays():
    w = tensor(512, 11008, 3, 0.05)
    lay, eager = (X.Mx4Linear(48, 512, 11008, BF16, "cuda", train=False) for _ in range(2))
    lay.set_weight(w)
    eager.set_weight(w)
    for m in (1, 17, 48):                # one launch, and the quantizer's beside it
        x, got = tensor(m, 512, m), []
        step = L.CapturedStep(lambda: got.append(lay.forward(x)))
        x.copy_(tensor(m, 512, 100 + m))
        step.replay()
        assert torch.equal(got[-1], eager.forward(x))


def test_two_blocks_on_two_streams():
    M, C, F = 1500, 700, 1100
    blocks = [block_of(M, C, F, 1), block_of(M, C, F, 5)]
    args = [[tensor(M, C, 10 * s + k) for k in range(4)] for s in (1, 2)]
    want = [[t.clone() for t in outputs(b, *a)] for b, a in zip(blocks, args)]
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for s in streams:
        s.wait_stream(torch.cuda.current_stream())
    for _ in range(5):
        got = []
        for s, b, a in zip(streams, blocks, args):
            with torch.cuda.stream(s):
                got.append(outputs(b, *a))
        torch.cuda.synchronize()
        for g, w in zip(got, want):
            assert all(torch.equal(p, q) for p, q in zip(g, w))
    assert all(b.status() == 0 for b in blocks)


def check(d, want, size, K):
    # FP32 sums of K exact products in any order: K - 1 roundings of 2^-24 of the sum of the
    # magnitudes, doubled for an accumulator that truncates; the output's rounding is monotone
    off = size * (K * 2.0 ** -23)
    low, high = (want - off).to(d.dtype).double(), (want + off).to(d.dtype).double()
    assert ((low <= d.double()) & (d.double() <= high)).all()


# 56 to 64 tiles of 256 x 256 in each of the three products: CTA pairs, with ragged last tiles
@pytest.mark.parametrize("dtype", [torch.float32, BF16])
@pytest.mark.parametrize("M,K,Nn", [(1600, 1800, 1904), (1601, 1795, 1901)])
def test_a_layer_of_paired_tiles(M, K, Nn, dtype):
    lay = X.Mx4Linear(M, K, Nn, dtype, "cuda")
    x, w, dy = (tensor(r, c, s, dtype=dtype) for r, c, s in ((M, K, 1), (K, Nn, 2), (M, Nn, 3)))
    lay.set_weight(w)
    y, (dx, dw) = lay.forward(x), lay.backward(dy, seed=11)
    assert lay.status.item() == 0
    xn, wn, gn = (t.double().cpu().numpy() for t in (x, w, dy))
    u = R.draws(M, Nn, 11)
    for got, a, b, k in ((y, R.mx4(xn), R.mx4(wn.T), K), (dx, R.mx4(gn, u), R.mx4(wn), Nn),
                         (dw, R.mx4(xn.T), R.mx4(gn.T, u.T), M)):
        a, b = torch.from_numpy(a).cuda(), torch.from_numpy(b).cuda()
        check(got, a @ b.t(), a.abs() @ b.abs().t(), k)

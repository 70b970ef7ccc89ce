"""Objects that share the buffers of what does not outlast a call's use: what a further MLP block of a
chain holds (CPU), and that a chain's results do not change (GPU)."""
import pytest
import torch

from paper_2411_10948_gb300 import build, microscale as X

BF16 = torch.bfloat16


@pytest.fixture(scope="module", autouse=True)
def library():
    build.build_library()


def storages(obj, seen=None):
    """{address: bytes} of every buffer that an object and its parts hold."""
    seen = {} if seen is None else seen
    for v in vars(obj).values():
        if isinstance(v, torch.Tensor):
            s = v.untyped_storage()
            if s.nbytes():
                seen[s.data_ptr()] = s.nbytes()
        elif hasattr(v, "__dict__") and type(v).__module__ == X.__name__:
            storages(v, seen)
    return seen


@pytest.mark.parametrize("gated", [True, False])
def test_a_further_block_holds_its_weights_and_what_it_keeps(gated):
    M, C, F = 1024, 256, 512
    up = 2 * F if gated else F
    first = X.Mx4MlpBlock(M, C, F, BF16, "cpu", gated=gated)
    more = X.Mx4MlpBlock(M, C, F, BF16, "cpu", gated=gated, share=first)
    old, new = storages(first), storages(more)
    own = sum(n for p, n in new.items() if p not in old)
    weights = C * up + F * C
    # 33 bytes per 32 elements of the norm's and the activation's inputs, 17 of the products'; a row's
    # statistics; both orientations of the weights' codes, and fp32 gradients
    kept = M * (C + up) * 33 // 32 + M * (C + F) * 17 // 32 + 8 * M
    assert own == kept + weights * 2 * 17 // 32 + 4 * weights + 4 * C + 4 * 4
    # less than the 16-bit inputs of the norm, the activation and both products
    assert kept < 0.55 * 2 * M * (C + up + C + F)
    # two objects that share nothing hold nothing in common
    apart = storages(X.Mx4MlpBlock(M, C, F, BF16, "cpu", gated=gated))
    assert not set(apart) & set(old) and sum(apart.values()) == sum(old.values())


def test_only_objects_made_alike_share():
    lay = X.Mx4Linear(64, 96, 32, BF16, "cpu")
    for args, train in (((63, 96, 32, BF16), True), ((64, 95, 32, BF16), True), ((64, 96, 31, BF16), True),
                        ((64, 96, 32, torch.float32), True), ((64, 96, 32, BF16), False)):
        with pytest.raises(ValueError):
            X.Mx4Linear(*args, "cpu", train=train, share=lay)
    act = X.Act8(64, 96, BF16, "silu", True, "cpu")
    X.Act8(64, 96, BF16, "gelu", True, "cpu", share=act)       # another activation has the same buffers
    for M, F, gated, train in ((63, 96, True, True), (64, 95, True, True), (64, 96, False, True), (64, 96, True, False)):
        with pytest.raises(ValueError):
            X.Act8(M, F, BF16, "silu", gated, "cpu", train=train, share=act)
    norm = X.Norm8(64, 96, BF16, "rms", "cpu", residual=True)
    X.Norm8(64, 96, BF16, "layer", "cpu", residual=True, share=norm)
    for M, C, residual, train in ((63, 96, True, True), (64, 95, True, True), (64, 96, False, True), (64, 96, True, False)):
        with pytest.raises(ValueError):
            X.Norm8(M, C, BF16, "rms", "cpu", residual=residual, train=train, share=norm)
    with pytest.raises(ValueError):
        X.Mx4MlpBlock(64, 96, 128, BF16, "cpu", share=X.Mx4MlpBlock(64, 96, 160, BF16, "cpu"))
    with pytest.raises(ValueError):
        X.Act8(64, 96, BF16, "silu", True, "meta", share=act)


def tensor(rows, cols, seed, scale=1.0):
    g = torch.Generator("cuda").manual_seed(seed)
    return (torch.randn((rows, cols), generator=g, device="cuda") * scale).to(BF16)


@pytest.mark.gpu
@pytest.mark.parametrize("M,C,F,rows", [(300, 256, 352, 300), (300, 256, 352, 77), (130, 65, 130, 130)])
def test_a_chain_gives_what_separate_blocks_give(M, C, F, rows):
    n = 4
    apart = [X.Mx4MlpBlock(M, C, F, BF16, "cuda") for _ in range(n)]
    chain = [X.Mx4MlpBlock(M, C, F, BF16, "cuda")]
    chain += [X.Mx4MlpBlock(M, C, F, BF16, "cuda", share=chain[0]) for _ in range(n - 1)]
    for k in range(n):
        gamma, w1, w2 = 1 + 0.1 * torch.randn(C, device="cuda"), tensor(C, 2 * F, k, 0.1), tensor(F, C, 10 + k, 0.1)
        apart[k].set_weights(gamma, w1, w2)
        chain[k].set_weights(gamma, w1, w2)
    delta, x, dout, dx = (tensor(rows, C, 20 + k) for k in range(4))

    def step(blocks):
        d, s = delta, x
        for b in blocks:
            d, s = b.forward(d, s)
        forward = d.clone(), s.clone()
        d, s = dout, dx
        for k in reversed(range(n)):
            d = s = blocks[k].backward(d, s, seed=2 * k)
        return (*forward, d.clone(), *(g for b in blocks for g in (b.dw1, b.dw2, b.dgamma)))

    for _ in range(2):
        for a, b in zip(step(apart), step(chain)):
            assert torch.equal(a, b)
    assert all(b.status() == 0 for b in chain)

"""A block divided among tensor-parallel ranks: the sums over their shares are the
whole block's result and gradients."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

if torch.cuda.is_available():
    from paper_2504_14145_amd.stage import Block


@pytest.fixture(autouse=True)
def need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


def near(got, want):
    """Roundings of every rank's partial result to 8 bits: 2^-6 of the norm, far below
    the residual or the bias once too often."""
    return float((got.double() - want.double()).norm()) <= 2.0 ** -6 * float(want.double().norm())


@pytest.mark.parametrize("tp,p", [(2, 0.0), (4, 0.3)])
def test_shares_add_up(tp, p):
    h, f, t = 128, 256, 70
    whole = Block(h, f, p=p, layer=2, seed=4)
    g = torch.Generator().manual_seed(1)
    whole.b1.copy_(torch.randn(f, generator=g) * 0.3)
    whole.b2.copy_(torch.randn(h, generator=g))
    whole.gamma.copy_(1 + 0.2 * torch.randn(h, generator=g))
    x, dy = (torch.randn((t, h), generator=g).bfloat16().cuda() for _ in range(2))
    want, saved = whole.forward(x, seed=9, row0=3)
    dx = whole.backward(dy, saved)
    y_sum, dx_sum, grads = 0, 0, {n: [] for n in whole.grads}
    for rank in range(tp):
        share = Block(h, f, p=p, layer=2, tp=tp, rank=rank)
        mine = slice(rank * f // tp, (rank + 1) * f // tp)
        share.w1.copy_(whole.w1[mine])
        share.b1.copy_(whole.b1[mine])
        share.w2.copy_(whole.w2[:, mine])
        share.b2.copy_(whole.b2)
        share.gamma.copy_(whole.gamma)
        y, saved = share.forward(x, seed=9, row0=3)
        y_sum, dx_sum = y_sum + y.float(), dx_sum + share.backward(dy, saved).float()
        for n, v in share.grads.items():
            grads[n].append(v)
    assert near(y_sum, want) and near(dx_sum, dx)
    assert near(torch.cat(grads["w1"]), whole.grads["w1"]) and near(torch.cat(grads["b1"]), whole.grads["b1"])
    assert near(torch.cat(grads["w2"], 1), whole.grads["w2"])
    for n in ("b2", "gamma", "beta"):
        assert near(sum(grads[n]), whole.grads[n]), n


def test_ranks_are_those_of_tp():
    for rank in (-1, 2):
        with pytest.raises(ValueError):
            Block(64, 128, tp=2, rank=rank)

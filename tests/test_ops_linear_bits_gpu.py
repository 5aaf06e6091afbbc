"""The gradient between dy and the products.  Where it is representable in 16 bits:
without an activation and with ReLU it is dy or 0, and dropout's factor is the
products', so nothing but the float32 sums and the result's rounding is left in dx and dw.
Where an element is dropped: 0, whatever pre holds.  Where pre is stored as an
infinity: the slope's limit."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from ops_reference import EPS32, assert_close, dot_bound, mask  # noqa: E402

if torch.cuda.is_available():
    from paper_2504_14145_amd import ops

BF16, F16 = torch.bfloat16, torch.float16


@pytest.fixture(autouse=True)
def need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


# whole tiles, ragged ones, and a contraction that is split
@pytest.mark.parametrize("m,n,k", [(128, 256, 192), (201, 131, 75), (2600, 40, 56)])
@pytest.mark.parametrize("act", ["none", "relu"])
@pytest.mark.parametrize("dtype", [BF16, F16], ids=str)
def test_gradients_of_a_dropout_keep_every_bit_of_dy(m, n, k, act, dtype):
    g = torch.Generator().manual_seed(m)
    x, dy, pre = (torch.randn(s, generator=g).to(dtype) for s in ((m, k), (m, n), (m, n)))
    w = (torch.randn((n, k), generator=g) * n ** -0.5).to(dtype)
    drop = ops.Dropout(0.1, 31, offset=2, row0=7)
    want_g = torch.where(mask(drop, m, n), dy.double(), 0.0)
    if act == "relu":
        want_g = torch.where(pre > 0, want_g, 0.0)
    args = dict(act=act, dropout=drop, pre=pre.cuda() if act != "none" else None)
    dx, dw, db = ops.linear_backward(dy.cuda(), x.cuda(), w.cuda(), **args)
    dw32 = torch.zeros((n, k), device="cuda")
    ops.linear_backward(dy.cuda(), x.cuda(), w.cuda(), **args, dw=dw32, bias=False, need_dx=False)
    for got, a, b, length, name in ((dx, want_g, w, n, "dx"), (dw, want_g.T, x, m, "dw"), (dw32, want_g.T, x, m, "dw32")):
        want, size = drop.scale * (a @ b.double()), drop.scale * (a.abs() @ b.double().abs())
        assert_close(got, want, dot_bound(length, size) + 2 * EPS32 * want.abs(), got.dtype, name)
    want, size = drop.scale * want_g.sum(0), drop.scale * want_g.abs().sum(0)
    assert_close(db, want, dot_bound(m, size), dtype, "db")


@pytest.mark.parametrize("act", ["relu", "silu", "gelu"])
def test_what_pre_holds_under_the_mask_does_not_matter(act):
    """NaN and infinities in pre at dropped places: the forward's result there is
    the residual, so the gradients are those of any finite pre."""
    m, n, k = 70, 88, 48
    g = torch.Generator().manual_seed(2)
    x, dy, pre = (torch.randn(s, generator=g).to(BF16) for s in ((m, k), (m, n), (m, n)))
    w = torch.randn((n, k), generator=g).to(BF16)
    drop = ops.Dropout(0.5, 3)
    keep = mask(drop, m, n)
    bad = pre.clone()
    for i, v in enumerate((float("nan"), float("inf"), float("-inf"))):
        at = torch.zeros((m, n), dtype=torch.bool)
        at[i::5] = True
        bad[at & ~keep] = v
    call = lambda p: ops.linear_backward(dy.cuda(), x.cuda(), w.cuda(), act=act, dropout=drop, pre=p.cuda())  # noqa: E731
    assert not bool(torch.isfinite(bad).all())
    for got, want in zip(call(bad), call(pre)):
        assert bool(torch.isfinite(want).all()) and torch.equal(got, want)


@pytest.mark.parametrize("act", ["relu", "silu", "gelu"])
def test_a_pre_beyond_the_types_range_has_the_slopes_limit(act):
    """float16 holds a finite -70000 as an infinity; the forward's result there is 0 and
    so is the gradient.  Far on the other side the slope is 1."""
    m, n, k = 40, 48, 8
    x = torch.ones((m, k), dtype=F16)
    w = torch.full((n, k), -10000.0, dtype=F16)
    w[::3] = 10000.0
    g = torch.Generator().manual_seed(1)
    dy = torch.randn((m, n), generator=g).to(F16)
    pre = torch.empty((m, n), dtype=F16, device="cuda")
    y = ops.linear(x.cuda(), w.cuda(), act=act, pre=pre)
    up = torch.zeros((m, n), dtype=torch.bool)
    up[:, ::3] = True
    assert bool((y.cpu()[~up] == 0).all()) and bool(torch.isinf(pre).all())
    _, dw, db = ops.linear_backward(dy.cuda(), x.cuda(), w.cuda(), act=act, pre=pre, need_dx=False)
    kept = torch.where(up, dy.double(), 0.0)
    assert_close(db, kept.sum(0), dot_bound(m, kept.abs().sum(0)), F16, "db")
    want = kept.T @ x.double()
    assert_close(dw, want, dot_bound(m, kept.abs().T @ x.double()), F16, "dw")

"""How far dw is off where the gradient passes one activation and x another: the matrix
instructions take g rounded to the type, and x as a rounded value and what that left off.

Terms of dw's sums have gradients of either sign, so squares add up: with S^2 the sum of
all (g x)^2, and e_g and e_x what rounding g and x shows relative to their norms, dw is off
by the square root of D^2 + e_g^2 S^2, D its own rounding, and with x rounded too by that of
D^2 + (e_g^2 + e_x^2) S^2.  The limit has a quarter of e_x^2.  The means of x, an eighth of
its square, make columns of dw go together, so there are 260 rows of it and more: their
squares' sum scatters by sqrt(2 / 260) of an eighth, a hundredth.  Sums' own errors are a
thousandth of all this.
"""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from kept_reference import unpack  # noqa: E402
from ops_reference import act, slope  # noqa: E402

if torch.cuda.is_available():
    from paper_2504_14145_amd import ops

BF16, F16 = torch.bfloat16, torch.float16


@pytest.fixture(autouse=True)
def need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


def exact(dy, x8, pre8, x_act, act_, scale=1.0):
    x = act(unpack(x8.values, x8.scales), x_act)
    g = dy.cpu().double() * slope(unpack(pre8.values, pre8.scales), act_)
    return g.T.contiguous() @ x * scale, g, x


def error(v, dtype):
    """What rounding v leaves off, relative to its norm."""
    return float((v.to(dtype).double() - v).norm() / v.norm())


# restored beside the other passes or, beyond 2^22 vectors, by itself; contractions whole and
# split; rows that end inside a vector
SIZES = [(300, 264, 520), (2000, 136, 320), (140, 1027, 301), (77, 515, 640), (8300, 4048, 264)]


@pytest.mark.parametrize("act_,x_act", [("gelu", "silu"), ("silu", "gelu"), ("gelu", "gelu")])
@pytest.mark.parametrize("dtype", [BF16, F16], ids=str)
@pytest.mark.parametrize("m,k,n", SIZES)
def test_dw_behind_two_activations(m, k, n, dtype, act_, x_act):
    g = torch.Generator(device="cuda").manual_seed(m)
    normal = lambda *s: torch.randn(s, generator=g, device="cuda").to(dtype)  # noqa: E731
    x8, pre8, w, dy = ops.pack8(normal(m, k)), ops.pack8(normal(m, n)), normal(n, k), normal(m, n)
    dx, dw, db = ops.linear_backward(dy, x8, w, act=act_, x_act=x_act, pre=pre8)
    want, gs, xs = exact(dy, x8, pre8, x_act, act_)
    size = float(((gs * gs).sum(1) * (xs * xs).sum(1)).sum())
    own = float(((want.to(dtype).double() - want) ** 2).sum())
    limit = (own + size * (error(gs, dtype) ** 2 + error(xs, dtype) ** 2 / 4)) ** 0.5
    off = float((dw.cpu().double() - want).norm())
    assert off <= limit, (off, limit)
    # the others, and dw added to, have the bits of calls without them
    assert torch.equal(dx, ops.linear_backward(dy, x8, w, act=act_, x_act=x_act, pre=pre8, need_dw=False)[0])
    assert torch.equal(dw, ops.linear_backward(dy, x8, w, act=act_, x_act=x_act, pre=pre8, need_dx=False, bias=False)[1])
    acc = torch.zeros((n, k), device="cuda")
    ops.linear_backward(dy, x8, w, act=act_, x_act=x_act, pre=pre8, bias=False, dw=acc, accumulate=True)
    assert torch.equal(acc.to(dtype), dw)
    # from a pre in 16 bits
    pre = ops.unpack8(pre8, dtype)
    assert torch.equal(dw, ops.linear_backward(dy, x8, w, act=act_, x_act=x_act, pre=pre)[1])


@pytest.mark.parametrize("m", [0, 1, 63, 65])
def test_few_rows(m):
    g = torch.Generator(device="cuda").manual_seed(m)
    normal = lambda *s: torch.randn(s, generator=g, device="cuda").to(BF16)  # noqa: E731
    x8, pre8, w, dy = ops.pack8(normal(m, 40)), ops.pack8(normal(m, 24)), normal(24, 40), normal(m, 24)
    d = ops.Dropout(0.25, 9)
    dx, dw, db = ops.linear_backward(dy, x8, w, act="gelu", x_act="silu", pre=pre8, dropout=d)
    kept = (ops.dropout_add(torch.ones_like(dy), d) != 0).cpu()
    want, _, _ = exact(torch.where(kept, dy.cpu(), 0), x8, pre8, "silu", "gelu", d.scale)
    size = (torch.where(kept, dy.cpu(), 0).double() * slope(unpack(pre8.values, pre8.scales), "gelu")).abs().T.contiguous() @ \
        act(unpack(x8.values, x8.scales), "silu").abs() * d.scale
    # g, dw and the slopes' arithmetic; x's second part is off by 2^-16
    bound = 2.0 ** -8 * (1.05 * size + want.abs()) + 2.0 ** -126
    assert bool(((dw.cpu().double() - want).abs() <= bound).all())


def test_in_a_graph():
    g = torch.Generator(device="cuda").manual_seed(1)
    normal = lambda *s: torch.randn(s, generator=g, device="cuda").to(BF16)  # noqa: E731
    z, pre, w, dy = normal(500, 136), normal(500, 200), normal(200, 136), normal(500, 200)

    def step():
        return ops.linear_backward(dy, ops.pack8(z), w, act="gelu", x_act="silu", pre=ops.pack8(pre))

    step()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step()
    for _ in range(3):
        z.normal_()
        dy.normal_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(step(), out))

"""Values at the ends of the types, kept in 8 bits and restored through an activation."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from kept_reference import F8, pack, unpack  # noqa: E402
from ops_reference import TINY, U, act  # noqa: E402

if torch.cuda.is_available():
    from paper_2504_14145_amd import ops

F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
TYPES = [F32, BF16, F16]


@pytest.fixture(autouse=True)
def need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


def ends(dtype):
    """The type's largest and lowest values, what rounds up beyond them, and small ones."""
    f = torch.finfo(dtype)
    x = torch.full((8, 64), 0.5, dtype=torch.double)
    x[:, 33:40] = torch.tensor([-3.0, -1.0, -0.25, 0.0, 0.25, 1.0, 3.0])
    x[0, 3], x[1, 4], x[2, 5], x[3, 6] = f.max, f.min, f.max * 0.99, f.min * 0.97
    x[4, 40], x[5, 41] = f.max, f.min
    x[6, :32], x[7, :32] = f.max, f.min
    return x.to(dtype)


@pytest.mark.parametrize("name", ["none", "relu", "silu", "gelu"])
@pytest.mark.parametrize("to", TYPES, ids=str)
@pytest.mark.parametrize("dtype", TYPES, ids=str)
def test_ends_through_an_activation(dtype, to, name):
    """What rounded up beyond float32's range is its largest value, before the activation
    too: SiLU and GELU of the lowest are 0, not NaN."""
    q, s = pack(ends(dtype))
    most = torch.finfo(F32).max
    z = unpack(q, s).clamp(-most, most)
    want = act(z, name)
    got = ops.unpack8(ops.Packed8(q.cuda(), s.cuda()), to, act=name).cpu().double()
    assert torch.isfinite(got).all()
    f = torch.finfo(to)
    want = want.clamp(f.min, f.max)
    limit = U[to] * want.abs() + (0 if name == "none" else 2e-6 * torch.where(want != 0, z.abs(), 0)) + TINY[to]
    assert bool(((got - want).abs() <= limit).all())


@pytest.mark.parametrize("name", ["silu", "gelu"])
@pytest.mark.parametrize("m,k,n", [(40, 64, 32), (300, 264, 136)])
def test_gradients_from_an_x_kept_at_the_ends(m, k, n, name):
    """x restored beside the other passes: a lowest value gives 0 to the sums of dw."""
    g = torch.Generator().manual_seed(m)
    z = torch.randn((m, k), generator=g).to(BF16)
    z[3, 5], z[m - 1, k - 1] = torch.finfo(BF16).min, torch.finfo(BF16).min
    w, dy, pre = (torch.randn(s, generator=g).to(BF16).cuda() for s in ((n, k), (m, n), (m, n)))
    x8 = ops.pack8(z.cuda())
    x = act(unpack(x8.values, x8.scales).clamp_min(-torch.finfo(F32).max), name)
    assert float(x[3, 5]) == 0 and torch.isfinite(x).all()
    for kw in ({}, {"act": "silu", "pre": ops.pack8(pre)}):
        dx, dw, db = ops.linear_backward(dy, x8, w, x_act=name, **kw)
        assert torch.isfinite(dx).all() and torch.isfinite(dw).all() and torch.isfinite(db).all()
        # the columns of the lowest values have the sums of the others
        y8 = ops.Packed8(x8.values.clone(), x8.scales)
        y8.values.view(torch.uint8)[3, 5] = 0
        y8.values.view(torch.uint8)[m - 1, k - 1] = 0
        assert torch.equal(dw, ops.linear_backward(dy, y8, w, x_act=name, **kw)[1])

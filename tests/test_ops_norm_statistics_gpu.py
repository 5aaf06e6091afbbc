"""Group norm's float32 statistics where a sample's first rows are unlike the
others: a zero row before values far from zero, an outlier, masked positions."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

if torch.cuda.is_available():
    from paper_2504_14145_amd import ops

U = 2.0 ** -24


@pytest.fixture(autouse=True)
def need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


# a slab a workgroup, short and long; many long slabs; chunks of a sample
@pytest.mark.parametrize("b,s,c,groups", [(1, 577, 120, 24), (1, 1024, 32, 1), (3, 4096, 8, 1), (520, 5000, 16, 1),
                                          (512, 16384, 8, 2), (2, 16384, 96, 8), (1, 70000, 4, 2), (1, 6000, 4104, 3)])
@pytest.mark.parametrize("first,rows,mean", [(300.0, 1, 0.0), (30.0, 1, 0.0), (0.0, 1, 300.0), (0.0, 70, 300.0),
                                             (1000.0, 5, -3.0)])
def test_first_rows_unlike_the_others(b, s, c, groups, first, rows, mean):
    """The variance is a sum of squares about means that are right to a float32
    rounding, added up by many threads whose roundings average out: within 16 u
    of rstd at any length.  The mean: 8 u of its size and the spread, one rounding
    of the result, a few of the sums and their joins.  The 64-bit form is taken on the
    CPU: torch's sums over two dimensions of such arrays on the GPU have differed from
    run to run by percents."""
    x = torch.randn((b, s, c), generator=torch.Generator(device="cuda").manual_seed(s), device="cuda") + mean
    x[:, :rows] = first
    per = c // groups
    x, y, got_mean, got_rstd = (t.cpu() for t in (x, *ops.group_norm(x, groups)))
    for at in range(0, b, 64):
        part = slice(at, min(b, at + 64))
        v = x[part].double().view(-1, s, groups, per)
        m = v.mean((1, 3))
        d = v - m[:, None, :, None]
        var = (d * d).mean((1, 3))
        rstd, std = 1 / torch.sqrt(var + 1e-5), torch.sqrt(var)
        off = ((got_rstd[part].double() - rstd) / rstd).abs().max()
        assert float(off) <= 16 * U, f"rstd off by {float(off) / U:.1f} u"
        off = (got_mean[part].double() - m).abs() / (m.abs() + std)
        assert float(off.max()) <= 8 * U, f"mean off by {float(off.max()) / U:.1f} u"
        want = d * rstd[:, None, :, None]
        limit = 20 * U * want.abs() + 10 * U * ((m.abs() + std) * rstd)[:, None, :, None]
        assert bool(((y[part].double().view_as(want) - want).abs() <= limit).all())


@pytest.mark.parametrize("s,huge", [(40, 1e25), (40, 1e30), (70000, 1e25), (70000, 1e30)])
def test_huge_values_are_not_nan(s, huge):
    """Squares beyond float32's range: an infinite variance, results of 0."""
    x = torch.full((1, s, 32), 1.0, device="cuda")
    x[0, ::2] = huge
    y, mean, rstd = ops.group_norm(x, 4)
    assert bool((rstd == 0).all()) and bool((y == 0).all()) and bool(torch.isfinite(mean).all())


@pytest.mark.parametrize("b,s,c,groups", [(3, 0, 4096, 1), (3, 0, 2056, 1), (2, 0, 8192, 2), (5, 0, 64, 8),
                                          (2, 0, 40000, 1), (4, 7, 0, 3), (4, 0, 0, 2)])
def test_statistics_of_nothing(b, s, c, groups):
    """Mean 0 and variance 0, whatever kernels and memory held before."""
    ops.group_norm(torch.full((64, 3, 4096), 5.0, device="cuda"), 1)
    mean, rstd = (torch.full((b, groups), float("nan"), device="cuda") for _ in range(2))
    x = torch.empty((b, s, c), device="cuda")
    ops.group_norm(x, groups, eps=0.25, mean=mean, rstd=rstd)
    assert bool((mean == 0).all()) and bool((rstd == 2).all())

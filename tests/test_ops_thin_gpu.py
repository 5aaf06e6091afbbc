"""dip_linear for few rows: counts of rows at which fragments are laid out in
another way, contractions that end inside a wave's part, a fragment or a vector,
and infinities that products with zeros must not reach."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from test_ops_linear_gpu import check  # noqa: E402

if torch.cuda.is_available():
    from paper_2504_14145_amd import ops

F16, BF16 = torch.float16, torch.bfloat16


@pytest.fixture(autouse=True)
def need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


@pytest.mark.parametrize("m", [1, 2, 7, 8, 9, 16])
@pytest.mark.parametrize("n,k", [(8, 8), (9, 7), (41, 64), (40, 513), (23, 1000), (16, 4100), (8200, 71)])
def test_rows_and_contractions(m, n, k):
    check(m, n, k, BF16 if m % 2 else F16, act="silu", residual=True, p=0.2, seed=m + k, backward=False)


@pytest.mark.parametrize("m", [1, 8, 12])
@pytest.mark.parametrize("k", [72, 77, 600])
def test_infinities_stay_in_their_rows(m, k):
    """Lanes without elements or rows of their own add nothing, 0 * inf least of all."""
    g = torch.Generator().manual_seed(k)
    x, w = (torch.randn(s, k, generator=g).to(BF16).cuda() for s in (m, 21))
    want = ops.linear(x, w)
    w[5, k - 1] = float("inf")
    x[m - 1, 0] = float("nan")
    got = ops.linear(x, w)
    rows = torch.ones(21, dtype=torch.bool, device="cuda")
    rows[5] = False
    assert torch.equal(got[:m - 1][:, rows], want[:m - 1][:, rows])
    assert bool(got[:m - 1, 5].isinf().all()) and bool(got[m - 1].isnan().all())

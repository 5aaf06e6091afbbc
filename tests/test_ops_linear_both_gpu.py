"""Both gradients of a product in one call, whose products may share a launch, against
each of them alone: the same bits."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

if torch.cuda.is_available():
    from paper_2504_14145_amd import ops

BF16, F16, F32 = torch.bfloat16, torch.float16, torch.float32


@pytest.fixture(autouse=True)
def need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


# whole, dx's contraction split, dw's, both, odd sizes with rows copied, one row, too large
# to share
SIZES = [(300, 520, 264), (140, 264, 5000), (5000, 264, 140), (2500, 136, 2500), (3001, 251, 2903), (1, 64, 64),
         (1201, 1795, 1027), (4096, 4096, 4096)]


@pytest.mark.parametrize("dtype", (BF16, F16))
@pytest.mark.parametrize("m,k,n", SIZES)
def test_both_have_the_bits_of_each(m, k, n, dtype):
    g = torch.Generator(device="cuda").manual_seed(m + n)
    normal = lambda *s: torch.randn(s, generator=g, device="cuda").to(dtype)  # noqa: E731
    x, w, dy, pre = normal(m, k), normal(n, k), normal(m, n), normal(m, n)
    for kw in ({}, {"act": "silu", "pre": pre, "dropout": ops.Dropout(0.3, 5, offset=1)}):
        dx, dw, db = ops.linear_backward(dy, x, w, **kw)
        assert torch.equal(dx, ops.linear_backward(dy, x, w, need_dw=False, bias=False, **kw)[0])
        assert torch.equal(dw, ops.linear_backward(dy, x, w, need_dx=False, bias=False, **kw)[1])
        for into in (F32, dtype):
            old = torch.randn((n, k), generator=g, device="cuda").to(into)
            one, two = old.clone(), old.clone()
            ops.linear_backward(dy, x, w, need_dx=False, bias=False, dw=one, accumulate=True, **kw)
            got, _, _ = ops.linear_backward(dy, x, w, bias=False, dw=two, accumulate=True, **kw)
            assert torch.equal(one, two) and torch.equal(got, dx)


@pytest.mark.parametrize("m,k,n", SIZES[:4])
def test_nothing_beyond_the_results_is_written(m, k, n):
    """Rows of padded arrays: what lies between and behind them stays."""
    g = torch.Generator(device="cuda").manual_seed(2)
    normal = lambda *s: torch.randn(s, generator=g, device="cuda").to(BF16)  # noqa: E731
    x, w, dy = normal(m, k), normal(n, k), normal(m, n)
    want = ops.linear_backward(dy, x, w, bias=False)
    wide_x = torch.full((m + 3, k + 13), 7.0, dtype=BF16, device="cuda")
    wide_w = torch.full((n + 3, k + 5), 7.0, dtype=BF16, device="cuda")
    ops.linear_backward(dy, x, w, bias=False, dx=wide_x[1:m + 1, 3:k + 3], dw=wide_w[2:n + 2, 1:k + 1])
    for wide, got, (r, c) in ((wide_x, want[0], (1, 3)), (wide_w, want[1], (2, 1))):
        rows, cols = got.shape
        assert torch.equal(wide[r:r + rows, c:c + cols], got)
        wide[r:r + rows, c:c + cols] = 7.0
        assert bool((wide == 7.0).all())


@pytest.mark.parametrize("m,k,n", SIZES[:4])
def test_captured_and_on_another_stream(m, k, n):
    g = torch.Generator(device="cuda").manual_seed(3)
    x, w, dy = (torch.randn(s, generator=g, device="cuda").to(BF16) for s in ((m, k), (n, k), (m, n)))
    dx, dw = torch.empty_like(x), torch.empty_like(w)
    ops.linear_backward(dy, x, w, bias=False, dx=dx, dw=dw)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        ops.linear_backward(dy, x, w, bias=False, dx=dx, dw=dw)
    for _ in range(3):
        dy.normal_()
        dx.zero_(), dw.zero_()
        graph.replay()
        torch.cuda.synchronize()
        want = ops.linear_backward(dy, x, w, bias=False)
        assert torch.equal(dx, want[0]) and torch.equal(dw, want[1])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = ops.linear_backward(dy, x, w, bias=False, stream=side)
    side.synchronize()
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])

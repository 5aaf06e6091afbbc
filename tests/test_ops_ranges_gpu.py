"""The stage operators at the edges of their kernels' ranges: the boundaries
between the ways a size is handled, sizes whose offsets pass 32 bits, and calls
on tensors of other streams."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from ops_reference import EPS32, U, act, assert_close  # noqa: E402
from test_ops_elementwise_gpu import check_norm  # noqa: E402
from test_ops_linear_gpu import check  # noqa: E402

if torch.cuda.is_available():
    import paper_2504_14145_amd as dip
    from paper_2504_14145_amd import ops

F32, F16, BF16 = torch.float32, torch.float16, torch.bfloat16


@pytest.fixture(autouse=True)
def need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


# ------------------------------------------------------------ linear

@pytest.mark.parametrize("m", [15, 16, 17, 31, 32, 33])
@pytest.mark.parametrize("n,k", [(40, 255), (41, 256), (8200, 33), (24, 2300)])
def test_few_rows(m, n, k):
    check(m, n, k, F16 if m % 2 else BF16, act="silu", residual=True, p=0.2, seed=m, backward=False)


def test_few_rows_of_a_large_weight():
    """17 to 32 rows go another way when w has more than 2^25 elements."""
    for m in (16, 20, 32):
        check(m, 8200, 4200, BF16, act="relu", seed=m, backward=False)


@pytest.mark.parametrize("k", [1, 8, 31, 63, 64, 65, 127, 128, 129, 191, 192, 193, 256, 257, 320, 321])
def test_contraction_lengths(k):
    """Every number of tiles below the ring's length, whole and not, in all three
    products: k is the forward's contraction, n the input gradient's, m the
    weight's."""
    check(k + 32, 70, k, BF16, seed=k)
    check(70, k, 72, F16, seed=k + 1)


def test_large_tiles_with_ragged_edges():
    check(4000, 4090, 2100, BF16, act="gelu", residual=True, seed=2)


def test_large_tiles_aligned():
    check(2048, 8192, 1024, F16, act="none", bias=False, p=0.0, seed=3)


def test_split_contractions_with_an_epilogue():
    check(64, 96, 8200, BF16, act="gelu", residual=True, p=0.3, seed=5, backward=False)
    check(8200, 72, 64, F16, act="silu", p=0.1, seed=6)
    check(50, 8200, 64, BF16, act="gelu", seed=7)


def test_accumulated_gradients_of_a_split():
    """A weight gradient that is both split and added to, in both types."""
    m, n, k = 9000, 40, 48
    g = torch.Generator().manual_seed(1)
    x, dy = (torch.randn(s, generator=g).to(BF16) for s in ((m, k), (m, n)))
    w = torch.zeros((n, k), dtype=BF16)
    want = dy.double().T @ x.double()
    mag = dy.double().abs().T @ x.double().abs()
    for dtype in (F32, BF16):
        dw = torch.full((n, k), 3.0, dtype=dtype, device="cuda")
        ops.linear_backward(dy.cuda(), x.cuda(), w.cuda(), need_dx=False, bias=False, dw=dw, db=None, accumulate=True)
        assert_close(dw, want + 3.0, 2 * (m + 8) * EPS32 * mag + 4 * EPS32 * (want.abs() + 3), dtype, str(dtype))


def test_one_row_and_one_column():
    for m, n, k in ((1, 5000, 9), (5000, 1, 9), (1, 1, 5000), (700, 1, 1), (1, 3, 1)):
        check(m, n, k, BF16, act="gelu", residual=True, p=0.5, seed=m + n)


def test_linear_beyond_32_bit_offsets():
    """2^31 and more elements of x, y and residual: rows near the end against the
    plain product, and the weight's gradient over all rows."""
    m, n, k = 540000, 4096, 8
    g = torch.Generator(device="cuda").manual_seed(1)
    x = torch.randn((m, k), generator=g, device="cuda").to(BF16)
    w = torch.randn((n, k), generator=g, device="cuda").to(BF16)
    r = torch.empty((m, n), dtype=BF16, device="cuda").normal_(generator=g)
    assert m * n > 1 << 31
    drop = ops.Dropout(0.25, 5, row0=77)
    y = ops.linear(x, w, dropout=drop, residual=r)
    for at in (0, 262144, 524287, 539000, m - 40):
        rows = slice(at, at + 40)
        part = ops.linear(x[rows], w, dropout=ops.Dropout(0.25, 5, row0=77 + at), residual=r[rows])
        assert torch.equal(y[rows], part), at
    del y
    dx, dw, db = ops.linear_backward(r, x, w)
    for at in (0, 524287, m - 40):
        rows = slice(at, at + 40)
        want = r[rows].double() @ w.double()
        mag = r[rows].double().abs() @ w.double().abs()
        assert_close(dx[rows], want.cpu(), (2 * (n + 8) * EPS32 * mag).cpu(), BF16, f"dx {at}")
    want, mag, total = (torch.zeros(s, dtype=torch.double, device="cuda") for s in ((n, k), (n, k), (n,)))
    for at in range(0, m, 45000):
        rr, xx = r[at:at + 45000].double(), x[at:at + 45000].double()
        want += rr.t().contiguous() @ xx
        mag += rr.abs().t().contiguous() @ xx.abs()
        total += rr.sum(0)
    # sums of m terms in a tree of chunks: 2^13 in a row at most
    assert_close(dw, want.cpu(), 2 * 8192 * EPS32 * mag.cpu(), BF16, "dw")
    assert_close(db, total.cpu(), 2 * 8192 * EPS32 * r.double().abs().sum(0).cpu(), BF16, "db")


def test_strided_rows_beyond_32_bit_offsets():
    """A few rows of a very wide array: x and y start gigabytes apart."""
    n, k = 64, 72
    wide = torch.empty((1100, 1 << 21), dtype=BF16, device="cuda")
    x = wide[:, 5:5 + k]
    x.copy_(torch.randn((1100, k), device="cuda"))
    y = wide[:, 4096:4096 + n]
    w = torch.randn((n, k), device="cuda").to(BF16)
    ops.linear(x, w, out=y)
    assert torch.equal(y, ops.linear(x.contiguous(), w))


# ------------------------------------------------------------ dropout

def test_dropout_beyond_32_bits():
    m, n = 70000, 32768
    x = torch.ones((m, n), dtype=BF16, device="cuda")
    assert m * n > 1 << 31
    y = ops.dropout_add(x, ops.Dropout(0.4, 3))
    for at in (0, 65535, 65536, m - 9):
        part = ops.dropout_add(x[at:at + 9], ops.Dropout(0.4, 3, row0=at))
        assert torch.equal(y[at:at + 9], part), at


def test_dropout_of_more_items_than_a_launch_takes():
    """2^31 groups of eight columns and more: one column a row."""
    m = (1 << 31) - 20000
    x = torch.ones((m, 1), dtype=F16, device="cuda")
    y = ops.dropout_add(x, ops.Dropout(0.5, 4))
    for at in (0, 1 << 30, m - 100):
        assert torch.equal(y[at:at + 100], ops.dropout_add(x[at:at + 100], ops.Dropout(0.5, 4, row0=at))), at
    big = torch.ones((300000, 57600), dtype=F16, device="cuda")   # 2.16e9 items
    y = ops.dropout_add(big, ops.Dropout(0.5, 4))
    for at in (0, 298261, 298262, 299990):
        assert torch.equal(y[at:at + 10], ops.dropout_add(big[at:at + 10], ops.Dropout(0.5, 4, row0=at))), at


# ------------------------------------------------------------ group norm

@pytest.mark.parametrize("per", [511, 512, 513, 1024, 1025, 2048, 2049, 4096, 4097, 8192, 8193, 16384, 16391])
@pytest.mark.parametrize("dtype", [F32, BF16], ids=str)
def test_row_lengths(per, dtype):
    check_norm(3, 1, per, 1, dtype, "silu", seed=per)


@pytest.mark.parametrize("b,s,c,groups", [(2, 1, 140000, 70000), (70000, 2, 8, 2), (2, 3, 9000, 1), (1, 2, 8192, 2),
                                          (1, 4096, 8, 1), (1, 4097, 8, 1), (40, 64, 64, 32), (600, 100, 16, 1),
                                          (1, 70000, 4, 2), (2, 5000, 264, 33), (3, 64, 4104, 3), (1, 3, 2056, 257)])
def test_norm_regimes(b, s, c, groups):
    check_norm(b, s, c, groups, BF16, "silu", seed=c)


def test_norm_beyond_32_bit_offsets():
    b, s, c, groups = 1, 8400000, 256, 8
    x = torch.empty((b, s, c), dtype=BF16, device="cuda").normal_(0.5, 1.0)
    assert x.numel() > 1 << 31
    gamma, beta = (torch.randn(c, device="cuda").to(BF16) for _ in range(2))
    y, mean, rstd = ops.group_norm(x, groups, gamma, beta, act="silu")
    v = x.view(s, groups, -1)
    total, square = torch.zeros(groups, dtype=torch.double, device="cuda"), torch.zeros(groups, dtype=torch.double, device="cuda")
    for at in range(0, s, 200000):
        t = v[at:at + 200000].double()
        total += t.sum((0, 2))
        square += (t * t).sum((0, 2))
    count = s * (c // groups)
    want_mean = total / count
    want_rstd = 1 / torch.sqrt(square / count - want_mean ** 2 + 1e-5)
    assert torch.allclose(mean[0].double(), want_mean, rtol=0, atol=1e-5)
    assert torch.allclose(rstd[0].double(), want_rstd, rtol=1e-5)
    for at in (0, 4200000, s - 50):
        xh = ((x[0, at:at + 50].double().view(50, groups, -1) - mean[0].double()[:, None]) * rstd[0].double()[:, None]).view(50, c)
        z = xh * gamma.double() + beta.double()
        assert_close(y[0, at:at + 50], act(z, "silu").cpu(), (8 * EPS32 * (xh.abs() * gamma.double().abs() + 4 + z.abs()) + 4e-6 * z.abs()).cpu(),
                     BF16, f"y {at}")
    dx, dgamma, dbeta = ops.group_norm_backward(y, x, mean, rstd, groups, gamma, beta, act="none")
    want = torch.zeros(c, dtype=torch.double, device="cuda")
    for at in range(0, s, 200000):
        want += y[0, at:at + 200000].double().sum(0)
    assert torch.allclose(dbeta.double(), want, rtol=2 * U[BF16], atol=1.0)
    assert bool(torch.isfinite(dx[0, -1]).all()) and bool(torch.isfinite(dgamma).all())


def test_norm_carries_nan_and_infinity_of_its_own_group_only():
    x = torch.randn((2, 40, 32), device="cuda")
    want = ops.group_norm(x, 4)[0]
    x[0, 3, 9] = float("nan")
    x[1, 7, 30] = float("inf")
    y = ops.group_norm(x, 4)[0]
    bad = torch.zeros((2, 4), dtype=torch.bool)
    bad[0, 1] = bad[1, 3] = True
    y, want = y.view(2, 40, 4, 8).cpu(), want.view(2, 40, 4, 8).cpu()
    for i in range(2):
        for g in range(4):
            if bad[i, g]:
                assert bool(torch.isnan(y[i, :, g]).any())
            else:
                assert torch.equal(y[i, :, g], want[i, :, g])
    x = torch.randn((6, 1, 64), device="cuda")
    want = ops.group_norm(x, 1)[0]
    x[2, 0, 5] = float("nan")
    y = ops.group_norm(x, 1)[0]
    assert bool(torch.isnan(y[2]).all()) and torch.equal(y[torch.arange(6) != 2], want[torch.arange(6) != 2])


# ------------------------------------------------------------ streams

def test_workspaces_of_another_stream_are_not_given_away():
    """A call on a side stream while the current stream keeps allocating: its
    workspace, which torch's allocator gave to the current stream, stays its own."""
    m, n, k = 4096, 512, 515
    x, w = (torch.randn(s, device="cuda").to(BF16) for s in ((m, k), (n, k)))
    pre = torch.randn((m, n), device="cuda").to(BF16)
    dy = torch.randn((m, n), device="cuda").to(BF16)
    want = ops.linear_backward(dy, x, w, act="gelu", pre=pre)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    for _ in range(5):
        got = [torch.empty_like(t) for t in want]
        side.wait_stream(torch.cuda.current_stream())
        ops.linear_backward(dy, x, w, act="gelu", pre=pre, dx=got[0], dw=got[1], db=got[2], stream=side)
        for size in (1 << 20, 1 << 22, 1 << 24):
            torch.full((size,), -1.0, device="cuda")
        side.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(want, got))


def test_a_raw_stream_handle_is_a_stream_too():
    x = torch.randn((64, 72), device="cuda").to(BF16)
    w = torch.randn((40, 72), device="cuda").to(BF16)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    out = torch.empty((64, 40), dtype=BF16, device="cuda")
    side.wait_stream(torch.cuda.current_stream())
    ops.linear(x, w, out=out, stream=side.cuda_stream)
    side.synchronize()
    assert torch.equal(out, ops.linear(x, w))


def test_sizes_beyond_the_index_range_are_refused():
    x = torch.empty((4, 64), dtype=BF16, device="cuda")
    wide = x.as_strided((1, 64), (64, 1))
    assert ops.linear(wide, x[:, :]).shape == (1, 4)
    with pytest.raises(dip.DipSimError) as e:
        ops.linear(torch.empty((2, 64), dtype=BF16, device="cuda").as_strided((1, 64), (1, 1)).expand(3, 64), x)
    assert e.value.code == dip.E_INVAL      # rows that overlap

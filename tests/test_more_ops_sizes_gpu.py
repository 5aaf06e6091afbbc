"""Norm, rotary positions and 8-bit values at sizes beyond one launch and beyond 32-bit
offsets: what is repeated gives the same over and over."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

if torch.cuda.is_available():
    from paper_2504_14145_amd import ops

BF16, F8 = torch.bfloat16, torch.float8_e4m3fn


@pytest.fixture(autouse=True)
def memory_back():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    yield
    torch.cuda.empty_cache()


def repeated(times, t):
    out = torch.empty((times * t.shape[0], *t.shape[1:]), dtype=t.dtype, device="cuda")
    out.view(times, *t.shape).copy_(t.expand(times, *t.shape))
    return out


def same(got, want):
    """Every one of the repetitions, in pieces that leave memory for the rest."""
    got = got.view(-1, *want.shape)
    if got.dtype is F8:
        got, want = got.view(torch.uint8), want.view(torch.uint8)
    return all(bool((g == want).all()) for g in got.split(1 << 16))


@pytest.mark.parametrize("m,c", [((1 << 29) + 4096, 8), ((1 << 21) + 4096, 1032), ((1 << 17) + 4096, 17000)])
def test_norm(m, c):
    g = torch.Generator(device="cuda").manual_seed(1)
    x1, r1, dy1 = (torch.randn((4096, c), generator=g, device="cuda").to(BF16) for _ in range(3))
    w = torch.randn(c, generator=g, device="cuda").to(BF16)
    times = m // 4096
    wy, wt, ws, wp = ops.rms_norm(x1, w, residual=r1, packed=True)
    x, r = repeated(times, x1), repeated(times, r1)
    y, total, rstd, p = ops.rms_norm(x, w, residual=r, total=r, packed=True)
    assert same(y, wy) and same(total, wt) and same(rstd, ws) and same(p.values, wp.values) and same(p.scales, wp.scales)
    del y, p
    dy = x.view(times, 4096, c).copy_(dy1.expand(times, 4096, c)).view(m, c)
    wdx, wdg = ops.rms_norm_backward(dy1, wt, ws, w, dtotal=r1, dgamma=torch.zeros(c, device="cuda"), accumulate=True)
    dt = repeated(times, r1)
    dx, dg = ops.rms_norm_backward(dy, total, rstd, w, dtotal=dt, dx=dt, dgamma=torch.zeros(c, device="cuda"), accumulate=True)
    assert same(dx, wdx)
    # Rows that repeat with the workgroups' stride: a thread adds one value up to 4097
    # times, and roundings of such a sum all go one way.  Chains of that many, of a
    # workgroup's 64 rows and of 2048 workgroups by sixteens are 4097 + 64 + 128 + 16
    # additions, each off by at most 2^-24 of the sum of magnitudes.
    size = (dy1.float() * wt.float() * ws[:, None]).abs().sum(0) * times
    assert bool(((dg - wdg * times).abs() <= (4097 + 64 + 128 + 16) * 2.0 ** -24 * size).all())


def test_packing_of_more_rows_than_a_launch_takes():
    x1 = torch.randn((4096, 1), device="cuda").to(BF16)
    want = ops.pack8(x1)
    p = ops.pack8(repeated((1 << 17) + 1, x1))
    assert same(p.values, want.values) and same(p.scales, want.scales)
    back = ops.unpack8(p)
    assert same(back, ops.unpack8(want))


def test_restoring_beyond_a_launch_and_32_bits():
    x1 = torch.randn((4096, 9), device="cuda").to(BF16)
    one = ops.pack8(x1)
    p = ops.Packed8(repeated((1 << 18) + 1, one.values.view(torch.uint8)).view(F8), repeated((1 << 18) + 1, one.scales))
    assert same(ops.unpack8(p, act="gelu"), ops.unpack8(one, act="gelu"))


@pytest.mark.parametrize("interleaved", [False, True])
def test_rotary(interleaved):
    t = (1 << 25) + 4096
    g = torch.Generator(device="cuda").manual_seed(2)
    q1 = torch.randn((4096, 60, 2), generator=g, device="cuda").to(BF16)
    k1 = torch.randn((4096, 4, 2), generator=g, device="cuda").to(BF16)
    pos1 = torch.randint(0, 1 << 20, (4096, 2), generator=g, device="cuda")
    freq, axis = ops.rotary_frequencies((0, 1))
    want, wk = ops.rotary(q1, pos1, freq, axis, k=k1, interleaved=interleaved)
    q, k, pos = (repeated(t // 4096, v) for v in (q1, k1, pos1))
    out, ok = ops.rotary(q, pos, freq, axis, k=k, interleaved=interleaved, out=q)
    assert out is q and same(q, want) and same(ok, wk)


def test_kept_products_beyond_32_bit_offsets():
    g = torch.Generator(device="cuda").manual_seed(3)
    m, n = (1 << 17) + 300, 16500
    x, w = torch.randn((m, 64), generator=g, device="cuda").to(BF16), torch.randn((n, 64), generator=g, device="cuda").to(BF16)
    pre = ops.Packed8.empty(m, n)
    y = ops.linear(x, w, act="relu", pre=pre)
    few = ops.Packed8.empty(300, n)
    wy = ops.linear(x[-300:], w, act="relu", pre=few)
    assert torch.equal(y[-300:], wy) and torch.equal(pre.scales[-300:], few.scales)
    assert torch.equal(pre.values[-300:].view(torch.uint8), few.values.view(torch.uint8))
    # the other way round: that array as x, and as pre
    dy = torch.randn((m, 64), generator=g, device="cuda").to(BF16)
    v = torch.randn((64, n), generator=g, device="cuda").to(BF16)
    got = ops.linear_backward(dy, pre, v, bias=False, need_dx=False)[1]
    assert torch.equal(got, ops.linear_backward(dy, ops.unpack8(pre), v, bias=False, need_dx=False)[1])
    grad = lambda rows, kept: ops.linear_backward(y[rows], x[rows], w, act="silu", pre=kept, bias=False,  # noqa: E731
                                                  need_dw=False)[0]
    whole, last = slice(0, m), slice(m - 300, m)
    dx, far = grad(whole, pre), grad(last, few)
    assert torch.equal(dx, grad(whole, ops.unpack8(pre)))
    # the last rows alone, whose sum over n is cut otherwise: two float32 sums of the same
    # n products, each within 2 (n + 8) 2^-24 of their magnitudes, and two roundings of 2^-8
    z = ops.unpack8(few, torch.float32).double()
    s = torch.sigmoid(z)
    size = (y[last].double() * s * (1 + z * (1 - s))).abs() * (1 + 2.0 ** -8) @ w.double().abs()
    limit = 4 * (n + 8) * 2.0 ** -24 * size
    limit = limit + 2 * 2.0 ** -8 * (far.double().abs() + limit)
    assert bool(((dx[last].double() - far.double()).abs() <= limit).all())

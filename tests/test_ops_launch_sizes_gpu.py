"""Sizes that the checks accept and that one launch has no threads for."""
import ctypes

import pytest

torch = pytest.importorskip("torch")

import paper_2504_14145_amd as dip  # noqa: E402
from paper_2504_14145_amd import ops  # noqa: E402

BF16 = torch.bfloat16
gpu = pytest.mark.gpu


@pytest.fixture(autouse=True)
def memory_back():
    yield
    if torch.cuda.is_available():
        torch.cuda.empty_cache()


@pytest.mark.parametrize("m,n,k,code", [((1 << 31) - 1, 256, 8, dip.E_CAPACITY), ((1 << 31) - 1, 257, 8, dip.E_RANGE),
                                        (16, 1 << 22, 1 << 18, dip.E_RANGE), ((1 << 31) - 1, 8, 264, dip.E_RANGE)])
def test_products_beyond_a_launch_are_refused(m, n, k, code):
    """More tiles than a grid has; at the limit only the missing workspace counts."""
    at = 1 << 20
    a = ops._Linear(m=m, n=n, k=k, dtype=ops.BF16, x=at + 2, ldx=k, w=at, ldw=k, y=at, ldy=n)
    assert ops._load().dip_linear(ctypes.byref(a), None) == code


def repeated(rows, t):
    """t over and over, to `rows` times its samples."""
    out = torch.empty((rows * t.shape[0], *t.shape[1:]), dtype=t.dtype, device="cuda")
    out.view(rows, *t.shape).copy_(t.expand(rows, *t.shape))
    return out


@gpu
@pytest.mark.parametrize("b,s,c,groups", [(1 << 24, 2, 8, 2), (1 << 29, 1, 8, 1), (1 << 24, 1, 1032, 1)])
def test_norm_of_more_samples_than_a_launch_takes(b, s, c, groups):
    """4096 samples over and over: every one as the first ones, which a small call
    gives too."""
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    g = torch.Generator(device="cuda").manual_seed(1)
    one = torch.randn((4096, s, c), generator=g, device="cuda").to(BF16)
    gamma, beta = (torch.randn(c, generator=g, device="cuda").to(BF16) for _ in range(2))
    want, wm, wr = ops.group_norm(one, groups, gamma, beta, act="silu")
    x = repeated(b // 4096, one)
    y, mean, rstd = ops.group_norm(x, groups, gamma, beta, act="silu")
    assert bool((y.view(-1, *one.shape) == want).all())
    assert bool((mean.view(-1, *wm.shape) == wm).all()) and bool((rstd.view(-1, *wr.shape) == wr).all())
    del y
    dwant, gw, bw = ops.group_norm_backward(one, one, wm, wr, groups, gamma, beta, act="silu")
    dx, dgamma, dbeta = ops.group_norm_backward(x, x, mean, rstd, groups, gamma, beta, act="silu")
    assert bool((dx.view(-1, *one.shape) == dwant).all())
    # both rounded to 8 bits; sums of up to 2^29 equal parts in float32, in some 2^13 to
    # 2^20 steps whose roundings are random: 2^-24 2^10 of their size
    for got, part in ((dgamma, gw), (dbeta, bw)):
        part = part.double() * (b // 4096)
        assert torch.allclose(got.double(), part, rtol=2.0 ** -7, atol=float(part.abs().max()) * 2.0 ** -7)


@gpu
def test_a_product_of_as_many_rows_as_there_are():
    m = (1 << 31) - 1
    x = torch.empty((m, 1), dtype=BF16, device="cuda")
    x.copy_(torch.arange(m, device="cuda", dtype=torch.int32).remainder_(251).unsqueeze(1))
    w = torch.tensor([[3.0]], dtype=BF16, device="cuda")
    y = ops.linear(x, w)
    for at in range(0, m, 1 << 28):
        part = slice(at, min(m, at + (1 << 28)))
        assert bool((y[part] == (x[part].float() * 3).to(BF16)).all())


@gpu
def test_packing_more_than_a_launch_takes():
    """2^35 elements of rows that start at odd addresses."""
    rows, k = 1 << 24, 2049
    g = torch.Generator(device="cuda").manual_seed(1)
    one = torch.randn((4096, k), generator=g, device="cuda").to(BF16)
    w = torch.randn((3, k), generator=g, device="cuda").to(BF16)
    x = repeated(rows // 4096, one)
    assert x.numel() >= 1 << 35
    y = ops.linear(x, w).view(-1, 4096, 3)
    assert bool((y == y[:1]).all())
    want = one.float() @ w.float().t().contiguous()
    # bf16's rounding, and float32 sums in two orders
    assert bool(((y[0].float() - want).abs() <= 2.0 ** -8 * want.abs() + 1e-3).all())

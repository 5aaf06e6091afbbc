"""Orders and strides other than a contiguous array's: the same values, the same
bits."""
import pytest

torch = pytest.importorskip("torch")

import paper_2504_14145_amd as dip  # noqa: E402
from paper_2504_14145_amd import ops  # noqa: E402

AT = 1 << 20     # an address that is never read
BF16 = torch.bfloat16
gpu = pytest.mark.gpu


@pytest.mark.parametrize("b,s,sb,ss,code", [
    (3, 5, 12, 36, dip.OK), (3, 5, 12, 35, dip.E_INVAL), (3, 5, 60, 12, dip.OK), (3, 5, 59, 12, dip.E_INVAL),
    (3, 5, 13, 38, dip.OK), (3, 5, 12, 12, dip.E_INVAL), (1, 5, 0, 12, dip.OK), (3, 1, 12, 0, dip.OK),
    (3, 1, 12, 1 << 60, dip.OK), (1, 5, 1 << 60, 12, dip.OK), (3, 5, 11, 36, dip.E_INVAL),
    (3, 5, (1 << 46) + 1, 12, dip.E_RANGE), (3, 5, 12, (1 << 46) + 1, dip.E_RANGE),
    ((1 << 31) - 1, 2, 1 << 46, 12, dip.OK), ((1 << 31) - 1, 2, 12, 1 << 35, dip.OK),
    ((1 << 31) - 1, 2, 12, 1 << 34, dip.E_INVAL)])
def test_which_strides_are_taken(b, s, sb, ss, code):
    import ctypes
    a = ops._GroupNorm(b=b, s=s, c=12, groups=1, dtype=ops.F16, eps=1e-5, x=AT, x_sb=sb, x_ss=ss, y=AT, y_sb=sb, y_ss=ss)
    need = ops._load().dip_group_norm_workspace(ctypes.byref(a))
    assert (need >= 0) if code == dip.OK else need == code


@gpu
@pytest.mark.parametrize("b,s,c,groups", [(5, 40, 96, 8), (3, 900, 64, 4), (2, 3000, 264, 33), (7, 1, 64, 2), (1, 30, 24, 3)])
def test_positions_outside_samples(b, s, c, groups):
    """Arrays laid out [s][b][c], and every one of a call in another order."""
    g = torch.Generator(device="cuda").manual_seed(3)
    x, dy = (torch.randn((b, s, c), generator=g, device="cuda").to(BF16) for _ in range(2))
    gamma, beta = (torch.randn(c, generator=g, device="cuda").to(BF16) for _ in range(2))
    other = lambda t: t.transpose(0, 1).contiguous().transpose(0, 1)  # noqa: E731
    y, mean, rstd = ops.group_norm(x, groups, gamma, beta, act="silu")
    want = ops.group_norm_backward(dy, x, mean, rstd, groups, gamma, beta, act="silu")
    out = other(torch.zeros_like(x))
    ops.group_norm(other(x), groups, gamma, beta, act="silu", out=out)
    assert torch.equal(out, y)
    dx = other(torch.zeros_like(x))
    got = ops.group_norm_backward(dy, other(x), mean, rstd, groups, gamma, beta, act="silu", dx=dx)
    assert all(torch.equal(p, q) for p, q in zip(got, want))
    got = ops.group_norm_backward(other(dy), x, mean, rstd, groups, gamma, beta, act="silu")
    assert all(torch.equal(p, q) for p, q in zip(got, want))


@gpu
def test_strides_that_nothing_steps_over():
    x = torch.randn((6, 1, 64), device="cuda")
    want = ops.group_norm(x, 2)[0]
    assert torch.equal(ops.group_norm(x.as_strided((6, 1, 64), (64, 1 << 40, 1)), 2)[0], want)
    wide = torch.randn((1 << 23) + 200, device="cuda").to(BF16)
    row = wide.view(1, -1)[:, 3:3 + 72]          # one row, 2^23 elements to the next
    w = torch.randn((40, 72), device="cuda").to(BF16)
    y = ops.linear(row, w)
    assert torch.equal(y, ops.linear(row.contiguous(), w))
    dy = torch.randn((1, 40), device="cuda").to(BF16)
    assert all(torch.equal(p, q) for p, q in zip(ops.linear_backward(dy, row, w), ops.linear_backward(dy, row.contiguous(), w)))

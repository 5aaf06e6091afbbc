"""dgamma and dbeta added to float32 arrays, as a block sums them over pieces."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from ops_reference import EPS32, GroupNorm, assert_close  # noqa: E402
from test_ops_elementwise_gpu import norm_inputs  # noqa: E402

if torch.cuda.is_available():
    from paper_2504_14145_amd import ops
    from paper_2504_14145_amd.stage import Block

F32, F16, BF16 = torch.float32, torch.float16, torch.bfloat16


@pytest.fixture(autouse=True)
def need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


# narrow rows of one workgroup and of many, rows, a slab of one sample and of many, chunks
@pytest.mark.parametrize("b,s,c,groups", [(20, 1, 64, 1), (900, 1, 200, 2), (70, 1, 1800, 1), (1, 40, 96, 8),
                                          (3, 40, 96, 8), (2, 3000, 264, 33), (0, 5, 24, 2), (3, 0, 24, 2)])
@pytest.mark.parametrize("dtype", [F32, F16, BF16], ids=str)
def test_added_in_float32(b, s, c, groups, dtype):
    """Twice onto what the arrays hold: no rounding to the type in between."""
    x, gamma, beta, dy = norm_inputs(b, s, c, dtype, 3)
    gx, gg, gb, gdy = (t.cuda() for t in (x, gamma, beta, dy))
    _, mean, rstd = ops.group_norm(gx, groups, gg, gb, act="silu")
    dgamma, dbeta = torch.full((c,), 2.0, device="cuda"), torch.full((c,), -1.0, device="cuda")
    for _ in range(2):
        dx, got_g, got_b = ops.group_norm_backward(gdy, gx, mean, rstd, groups, gg, gb, act="silu", dgamma=dgamma,
                                                   dbeta=dbeta, accumulate=True)
        assert got_g is dgamma and got_b is dbeta
    plain = ops.group_norm_backward(gdy, gx, mean, rstd, groups, gg, gb, act="silu")
    assert torch.equal(plain[0], dx)
    if b * s == 0:
        assert bool((dgamma == 2).all()) and bool((dbeta == -1).all())
        return
    want = GroupNorm(x, groups, gamma, beta, 1e-5, "silu").grads(dy)
    for got, name, start in ((dgamma, "dgamma", 2.0), (dbeta, "dbeta", -1.0)):
        v, bound = want[name]
        assert_close(got, start + 2 * v, 2 * bound + 8 * EPS32 * (abs(start) + 2 * v.abs()), F32, name)


def test_given_arrays_and_refusals():
    x, gamma, beta, dy = (t.cuda() for t in norm_inputs(3, 40, 96, BF16, 3))
    _, mean, rstd = ops.group_norm(x, 8, gamma, beta)
    args = dy, x, mean, rstd, 8, gamma, beta
    want = ops.group_norm_backward(*args)
    given = torch.empty_like(gamma), torch.empty_like(beta)
    ops.group_norm_backward(*args, dgamma=given[0], dbeta=given[1])
    assert torch.equal(given[0], want[1]) and torch.equal(given[1], want[2])
    f = torch.zeros(96, device="cuda")
    for call in (lambda: ops.group_norm_backward(*args, accumulate=True),
                 lambda: ops.group_norm_backward(*args, dgamma=f, dbeta=f),
                 lambda: ops.group_norm_backward(*args, dgamma=given[0], dbeta=given[1], accumulate=True),
                 lambda: ops.group_norm_backward(dy, x, mean, rstd, 8, dgamma=f, accumulate=True),
                 lambda: ops.group_norm_backward(*args, dgamma=f[:48], dbeta=f, accumulate=True)):
        with pytest.raises(ValueError):
            call()


def test_pieces_of_a_block_sum_in_float32():
    """Every piece's dgamma and dbeta reach the block's gradients unrounded: 64 pieces
    of one row, whose gradients only differ from the 64-bit ones of the same
    arriving gradient by float32 roundings."""
    block = Block(128, 256, act="relu", seed=3)
    g = torch.Generator().manual_seed(5)
    x = torch.randn((64, 128), generator=g).to(BF16).cuda()
    dy = torch.randn((64, 128), generator=g).to(BF16).cuda()
    want = {n: torch.zeros(128, dtype=torch.double) for n in ("gamma", "beta")}
    size = {n: torch.zeros(128, dtype=torch.double) for n in ("gamma", "beta")}
    for i in range(64):
        rows = slice(i, i + 1)
        _, saved = block.forward(x[rows])
        n, mean, rstd, pre, u = saved[3]
        du, _, _ = ops.linear_backward(dy[rows], u, block.w2, bias=False, need_dw=False)
        dn, _, _ = ops.linear_backward(du, n, block.w1, act="relu", pre=pre, bias=False, need_dw=False)
        xh = (x[rows].cpu().double() - mean.cpu().double()) * rstd.cpu().double()
        for name, part in (("gamma", dn.cpu().double() * xh), ("beta", dn.cpu().double())):
            want[name] += part[0]
            size[name] += part[0].abs()
        block.backward(dy[rows], saved)
    for name in want:
        off = (block.grads[name].cpu().double() - want[name]).abs()
        assert bool((off <= (64 + 8) * EPS32 * size[name]).all()), name

"""dip_dropout_add and dip_group_norm with its gradient against their plain
64-bit forms."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from ops_reference import EPS32, GroupNorm, assert_close, mask  # noqa: E402

if torch.cuda.is_available():
    import paper_2504_14145_amd as dip
    from paper_2504_14145_amd import ops

F32, F16, BF16 = torch.float32, torch.float16, torch.bfloat16


@pytest.fixture(autouse=True)
def need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


def strided(t, pad, shift):
    rows, cols = t.shape
    flat = torch.full((shift + rows * (cols + pad) + 8,), float("nan"), dtype=t.dtype, device="cuda")
    v = flat[shift:shift + rows * (cols + pad)].view(rows, cols + pad)[:, :cols]
    v.copy_(t)
    return v


@pytest.mark.parametrize("dtype", [F32, F16, BF16], ids=str)
@pytest.mark.parametrize("m,n,pad,shift", [(1, 1, 0, 0), (3, 7, 0, 0), (40, 64, 0, 0), (17, 1000, 3, 1),
                                           (9, 72, 8, 8), (33, 41, 7, 0), (130, 16, 0, 2)])
@pytest.mark.parametrize("p", [0.0, 0.1, 0.75])
def test_dropout(m, n, pad, shift, p, dtype):
    g = torch.Generator().manual_seed(m * 31 + n)
    x, r = torch.randn((m, n), generator=g).to(dtype), torch.randn((m, n), generator=g).to(dtype)
    d = ops.Dropout(p, 123456789012345, offset=(5 << 32) + 6, row0=n)
    keep = mask(d, m, n)
    want = torch.where(keep, x.double() * d.scale, 0.0)
    gx, gr = strided(x, pad, shift), strided(r, pad, shift)
    out = torch.full((m, n + pad), 7.0, dtype=dtype, device="cuda")
    assert_close(ops.dropout_add(gx, d, gr, out=out[:, :n]), want + r.double(),
                 4 * EPS32 * (want.abs() + r.double().abs()), dtype, "y")
    assert bool((out[:, n:] == 7.0).all())
    dx = ops.dropout_add(gx, d)
    assert_close(dx, want, 2 * EPS32 * want.abs(), dtype, "dx")
    assert torch.equal(dx.cpu()[~keep], torch.zeros(int((~keep).sum()), dtype=dtype))


def test_dropout_rate_and_limits():
    x = torch.ones((512, 1024), device="cuda")
    for p in (0.01, 0.3, 0.9):
        y = ops.dropout_add(x, ops.Dropout(p, 7))
        dropped = float((y == 0).double().mean())
        assert abs(dropped - p) < 6 * (p * (1 - p) / x.numel()) ** 0.5 + 1e-5
    near = ops.Dropout(0.99999, 3)
    assert near.drop_of == 65535
    y = ops.dropout_add(x, near)
    assert set(y.unique().tolist()) <= {0.0, 65536.0}
    with pytest.raises(dip.DipSimError):
        ops.dropout_add(x, ops.Dropout(0.5, 1, row0=(1 << 32) - 511))
    ops.dropout_add(x, ops.Dropout(0.5, 1, row0=(1 << 32) - 512))
    for empty in (x[:0], x[:, :0]):
        assert ops.dropout_add(empty, near).shape == empty.shape


def test_dropout_removes_infinities_and_may_work_in_place():
    x = torch.full((64, 80), float("inf"), dtype=BF16, device="cuda")
    x[:, ::2] = float("nan")
    d = ops.Dropout(0.5, 9)
    keep = mask(d, 64, 80)
    r = torch.randn((64, 80)).to(BF16)
    y = ops.dropout_add(x, d, r.cuda()).cpu()
    assert torch.equal(y[~keep], r[~keep]) and not bool(torch.isfinite(y[keep]).any())
    x = torch.randn((64, 80)).to(BF16).cuda()
    want = ops.dropout_add(x, d)
    assert torch.equal(want, ops.dropout_add(x, d, out=x)) and torch.equal(want, x)


# ------------------------------------------------------------ group norm

def norm_inputs(b, s, c, dtype, seed, shift=0.5):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn((b, s, c), generator=g) * (1 + torch.rand((c,), generator=g)) + shift + torch.randn((c,), generator=g) * 0.5
    return (x.to(dtype), (1 + 0.2 * torch.randn((c,), generator=g)).to(dtype),
            (0.2 * torch.randn((c,), generator=g)).to(dtype), torch.randn((b, s, c), generator=g).to(dtype))


def place(t, pad_c, pad_s, shift):
    """The same values in a wider array whose other values are NaN."""
    b, s, c = t.shape
    ss, sb = c + pad_c, (s + pad_s) * (c + pad_c)
    flat = torch.full((shift + b * sb + 8,), float("nan"), dtype=t.dtype, device="cuda")
    v = flat[shift:shift + b * sb].view(b, s + pad_s, ss)[:, :s, :c]
    v.copy_(t)
    return v


def check_norm(b, s, c, groups, dtype, act_name="silu", affine=True, eps=1e-5, pads=(0, 0, 0), seed=1, shift=0.5):
    x, gamma, beta, dy = norm_inputs(b, s, c, dtype, seed, shift)
    gamma, beta = (gamma, beta) if affine else (None, None)
    ref = GroupNorm(x, groups, gamma, beta, eps, act_name)
    gx, gdy = place(x, *pads), place(dy, *pads)
    gg, gb = (t.cuda() if t is not None else None for t in (gamma, beta))
    y = place(torch.zeros_like(x), *pads)
    _, mean, rstd = ops.group_norm(gx, groups, gg, gb, eps, act=act_name, out=y)
    what = f"b {b} s {s} c {c} groups {groups} {dtype} {act_name}"
    assert_close(mean, ref.mean[..., 0], 2 * EPS32 * (ref.mean[..., 0].abs() + 1e-30)
                 + (ref.xh_bound.amax(2) / ref.rstd[..., 0]), F32, what + " mean")
    assert_close(rstd, ref.rstd[..., 0], ref.rstd[..., 0] * (1e-6 + ref.xh_bound.amax(2)), F32, what + " rstd")
    assert_close(y, ref.y, ref.y_bound, dtype, what + " y")
    dx = place(torch.zeros_like(x), *pads)
    _, dgamma, dbeta = ops.group_norm_backward(gdy, gx, mean, rstd, groups, gg, gb, act=act_name, dx=dx)
    want = ref.grads(dy)
    assert_close(dx, *want["dx"], dtype, what + " dx")
    assert (dgamma is None) == (not affine)
    if affine:
        assert_close(dgamma, *want["dgamma"], dtype, what + " dgamma")
        assert_close(dbeta, *want["dbeta"], dtype, what + " dbeta")


SHAPES = [(1, 1, 1, 1), (1, 1, 8, 2), (2, 3, 6, 3), (1, 64, 320, 32), (3, 37, 60, 4), (2, 16, 96, 32),
          (5, 1, 1000, 1), (300, 1, 64, 1), (70, 1, 1792, 1), (9, 1, 4096, 1), (4, 1, 24, 3), (1, 1200, 16, 16),
          (2, 700, 128, 32), (1, 5000, 8, 1), (2, 130, 512, 8), (1, 9, 5000, 1), (2, 33, 40, 8), (1, 2500, 130, 26)]


@pytest.mark.parametrize("dtype", [F32, F16, BF16], ids=str)
@pytest.mark.parametrize("b,s,c,groups", SHAPES)
def test_norm_shapes(b, s, c, groups, dtype):
    check_norm(b, s, c, groups, dtype, act_name=("none", "silu", "gelu", "relu")[(b + s + c) % 4 if (b + s + c) % 4 < 3 else 0],
               seed=b + s)


@pytest.mark.parametrize("act_name", ["none", "silu", "gelu"])
@pytest.mark.parametrize("affine", [False, True])
@pytest.mark.parametrize("eps", [1e-6, 0.1])
def test_norm_forms(act_name, affine, eps):
    check_norm(2, 50, 48, 6, BF16, act_name, affine, eps, seed=4)
    check_norm(40, 1, 256, 1, F32, act_name, affine, eps, seed=5)


@pytest.mark.parametrize("pads", [(8, 0, 0), (0, 3, 0), (8, 2, 8), (1, 0, 0), (3, 1, 1), (0, 0, 1)])
@pytest.mark.parametrize("b,s,c,groups", [(2, 40, 64, 8), (3, 5, 30, 3), (20, 1, 512, 1), (2, 600, 96, 4)])
def test_norm_strides_and_alignment(b, s, c, groups, pads):
    check_norm(b, s, c, groups, F16, "silu", pads=pads, seed=6)
    check_norm(b, s, c, groups, F32, "none", pads=pads, seed=7)


@pytest.mark.parametrize("b,s,c,groups", [(3, 1, 512, 1), (1, 900, 64, 8), (2, 40, 96, 12)])
def test_norm_of_values_far_from_zero(b, s, c, groups):
    """A mean of 300 deviations: a sum of squares without a shift would lose it."""
    check_norm(b, s, c, groups, F32, "none", seed=8, shift=300.0)


def test_norm_relu_and_its_gradient():
    """Compared where z is not within the rounding of 0, at which the slope jumps."""
    x, gamma, beta, dy = norm_inputs(2, 30, 64, F32, 3)
    ref = GroupNorm(x, 8, gamma, beta, 1e-5, "relu")
    y, mean, rstd = ops.group_norm(x.cuda(), 8, gamma.cuda(), beta.cuda(), act="relu")
    assert_close(y, ref.y, ref.y_bound, F32, "y")
    assert bool((ref.z.abs() > 1e-5).all())
    dx, dgamma, dbeta = ops.group_norm_backward(dy.cuda(), x.cuda(), mean, rstd, 8, gamma.cuda(), beta.cuda(), act="relu")
    want = ref.grads(dy)
    for name, got in (("dx", dx), ("dgamma", dgamma), ("dbeta", dbeta)):
        assert_close(got, *want[name], F32, name)


def test_norm_of_equal_values_is_beta():
    x = torch.full((2, 20, 32), 3.25, device="cuda")
    beta = torch.randn(32, device="cuda")
    y, mean, rstd = ops.group_norm(x, 4, torch.ones(32, device="cuda"), beta, eps=1e-5)
    assert torch.equal(y, beta.expand_as(y)) and bool((mean == 3.25).all())
    assert torch.allclose(rstd, torch.full_like(rstd, 1e5 ** 0.5))


def test_norm_gradient_against_differences():
    b, s, c, groups, name = 2, 12, 24, 4, "gelu"
    x, gamma, beta, dy = norm_inputs(b, s, c, F32, 9)
    _, mean, rstd = ops.group_norm(x.cuda(), groups, gamma.cuda(), beta.cuda(), act=name)
    grads = ops.group_norm_backward(dy.cuda(), x.cuda(), mean, rstd, groups, gamma.cuda(), beta.cuda(), act=name)
    base = [x.double(), gamma.double(), beta.double()]
    g = torch.Generator().manual_seed(2)
    for i, grad in enumerate(grads):
        d = torch.randn(base[i].shape, generator=g).double()
        loss = []
        for h in (1e-5, -1e-5):
            at = [v + h * d if j == i else v for j, v in enumerate(base)]
            loss.append((GroupNorm(at[0], groups, at[1], at[2], 1e-5, name).y * dy.double()).sum())
        want = float((loss[0] - loss[1]) / 2e-5)
        got = float((grad.cpu().double() * d).sum())
        size = float((grad.cpu().double().abs() * d.abs()).sum())
        assert abs(got - want) <= 1e-4 * size, (i, got, want)   # 2e-6-level slopes, differences of 1e-6


def test_norm_parts_streams_and_graph():
    b, s, c, groups = 2, 300, 64, 8
    x, gamma, beta, dy = (t.cuda() for t in norm_inputs(b, s, c, BF16, 2))

    def step(stream=None):
        y, mean, rstd = ops.group_norm(x, groups, gamma, beta, act="silu", stream=stream)
        return (y, mean, rstd, *ops.group_norm_backward(dy, x, mean, rstd, groups, gamma, beta, act="silu", stream=stream))

    want = step()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = step(side)
    side.synchronize()
    assert all(torch.equal(a, g) for a, g in zip(want, got))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = step()
    for _ in range(3):
        for t in held:
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, g) for a, g in zip(want, held))
        assert all(torch.equal(a, g) for a, g in zip(want, step()))
    dx, none, _ = ops.group_norm_backward(dy, x, want[1], want[2], groups, gamma, beta, act="silu", need_dparam=False)
    assert none is None and torch.equal(dx, want[3])
    none, dgamma, dbeta = ops.group_norm_backward(dy, x, want[1], want[2], groups, gamma, beta, act="silu", need_dx=False)
    assert none is None and torch.equal(dgamma, want[4]) and torch.equal(dbeta, want[5])


def test_norm_refusals_and_empty():
    x, gamma, beta, dy = (t.cuda() for t in norm_inputs(2, 5, 12, F32, 2))
    for call in (lambda: ops.group_norm(x, 5), lambda: ops.group_norm(x, 3, eps=-1.0)):
        with pytest.raises(dip.DipSimError) as e:
            call()
        assert e.value.code == dip.E_INVAL
    for call in (lambda: ops.group_norm(x, 3, gamma[:6]), lambda: ops.group_norm(x[0], 3),
                 lambda: ops.group_norm(x, 0), lambda: ops.group_norm(x.transpose(1, 2), 5),
                 lambda: ops.group_norm(x, 3, act="swish"), lambda: ops.group_norm(x.cpu(), 3),
                 lambda: ops.group_norm(x, 3, gamma.half()),
                 lambda: ops.group_norm_backward(dy, x.half(), None, None, 3)):
        with pytest.raises(ValueError):
            call()
    y, mean, rstd = ops.group_norm(x[:0], 3, gamma, beta)
    assert y.shape == (0, 5, 12) and mean.shape == (0, 3)
    dx, dgamma, dbeta = ops.group_norm_backward(dy[:0], x[:0], mean, rstd, 3, gamma, beta)
    assert dx.shape == (0, 5, 12) and not bool(dgamma.any()) and not bool(dbeta.any())
    y, mean, rstd = ops.group_norm(x[:, :0], 3, gamma, beta, eps=0.25)
    assert bool((mean == 0).all()) and bool((rstd == 2).all())
    dx, dgamma, dbeta = ops.group_norm_backward(dy[:, :0], x[:, :0], mean, rstd, 3, gamma, beta)
    assert not bool(dgamma.any()) and not bool(dbeta.any())

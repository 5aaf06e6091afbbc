"""linear with the value before its activation kept in 8 bits, and its gradients from
activations kept so, against the plain 64-bit form."""
import itertools

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from kept_reference import F8, assert_kept, kept_x, pack, unpack  # noqa: E402
from ops_reference import Linear, assert_close  # noqa: E402

if torch.cuda.is_available():
    from paper_2504_14145_amd import ops

BF16, F16 = torch.bfloat16, torch.float16
ACTS = ("none", "relu", "silu", "gelu")


@pytest.fixture(autouse=True)
def need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


def dev(t):
    return None if t is None else t.cuda()


def check(m, n, k, dtype, act="gelu", x_act="none", bias=True, residual=False, p=0.0, seed=1, pad=0, grad_type=None):
    g = torch.Generator().manual_seed(seed)
    normal = lambda s, scale=1.0: (torch.randn(s, generator=g) * scale).to(dtype)  # noqa: E731
    x, w = normal((m, k)), normal((n, k), max(k, 1) ** -0.5)
    b, r = normal((n,), 0.5) if bias else None, normal((m, n)) if residual else None
    dy = normal((m, n), 0.3)
    drop = ops.Dropout(p, seed * 77 + 5, offset=seed, row0=3) if p else None
    ref = Linear(x, w, b, r, act, drop)
    what = f"m {m} n {n} k {k} {dtype} {act} {x_act} p {p}"
    # forward
    scales = (n + 31) // 32
    q8 = torch.full((m, n + pad), 0x5a, dtype=torch.uint8, device="cuda")
    s8 = torch.full((m, scales + pad), 0x5b, dtype=torch.uint8, device="cuda")
    pre = ops.Packed8(q8.view(F8)[:, :n], s8[:, :scales])
    y = ops.linear(dev(x), dev(w), dev(b), act=act, dropout=drop, residual=dev(r), pre=pre)
    assert_close(y, ref.y, ref.y_bound, dtype, what + " y")
    assert_kept(pre.values, pre.scales, ref.z, ref.z_bound, what + " pre")
    assert bool((q8[:, n:] == 0x5a).all()) and bool((s8[:, scales:] == 0x5b).all())
    # gradients, x kept before its own activation
    zq, zs = pack(normal((m, k)))
    x64, xb = kept_x(zq, zs, x_act, dtype)
    kx = torch.full((m, k + pad), 0x5a, dtype=torch.uint8, device="cuda")
    kx[:, :k] = zq.cuda().view(torch.uint8)
    kept = ops.Packed8(kx.view(F8)[:, :k], zs.cuda())
    ref.x = x64
    gt = dtype if grad_type is None else grad_type
    dw, db = (torch.full(s, 0.25, dtype=gt, device="cuda") for s in ((n, k), (n,)))
    acc = grad_type is not None
    dx, _, _ = ops.linear_backward(dev(dy), kept, dev(w), act=act, dropout=drop, pre=pre if act != "none" else None,
                                   x_act=x_act, dw=dw, db=db, accumulate=acc)
    want = ref.grads(dy, unpack(pre.values, pre.scales) if act != "none" else None, dtype)
    d = torch.where(ref.keep, dy.double().abs() * ref.scale, 0.0) * 1.2
    add = 0.25 if acc else 0.0
    assert_close(dx, *want["dx"], dtype, what + " dx")
    assert_close(dw, want["dw"][0] + add, want["dw"][1] + d.T @ xb + 2.0 ** -23 * add, gt, what + " dw")
    assert_close(db, want["db"][0] + add, want["db"][1] + 2.0 ** -23 * add, gt, what + " db")
    return y


@pytest.mark.parametrize("dtype", [BF16, F16], ids=str)
@pytest.mark.parametrize("m,n,k", [(1, 1, 1), (1, 64, 64), (2, 8, 2048), (5, 100, 72), (16, 136, 1024), (17, 33, 65),
                                   (64, 256, 96), (65, 130, 200), (129, 257, 40), (255, 72, 511), (300, 520, 264), (513, 384, 1100),
                                   (260, 2100, 320), (96, 1024, 2048), (40, 48, 8192)])
def test_shapes(m, n, k, dtype):
    check(m, n, k, dtype, act=ACTS[(m + n + k) % 4], x_act=ACTS[(m + n) % 4], residual=bool(m % 2), seed=m)


@pytest.mark.parametrize("act,x_act,p", itertools.product(ACTS, ACTS, (0.0, 0.3)))
def test_activations(act, x_act, p):
    check(70, 90, 48, BF16, act=act, x_act=x_act, residual=True, p=p, seed=3)


@pytest.mark.parametrize("pad", [1, 3, 32])
def test_rows_of_wider_arrays(pad):
    check(37, 75, 61, F16, pad=pad, p=0.25, seed=9)
    check(200, 320, 128, BF16, pad=pad, seed=9)


@pytest.mark.parametrize("dtype", [BF16, F16], ids=str)
def test_accumulated_gradients(dtype):
    check(130, 150, 77, dtype, grad_type=torch.float32, x_act="silu", seed=5)


# 128 x 128 tiles one and two a CU, split, 256 x 256, 192 x 128
@pytest.mark.parametrize("m,n,k", [(300, 520, 264), (2000, 1500, 512), (64, 100, 4096), (4100, 2200, 256), (5000, 4096, 64),
                                   (1152, 3840, 512)])
def test_the_output_has_the_bits_of_the_call_without(m, n, k):
    """Tiles of every size, whole and split: keeping pre changes nothing else, and what
    is kept is what packing the float32 values would have kept."""
    g = torch.Generator().manual_seed(m)
    x, w = (torch.randn(s, generator=g).to(BF16).cuda() for s in ((m, k), (n, k)))
    b, r = torch.randn(n, generator=g).to(BF16).cuda(), torch.randn((m, n), generator=g).to(BF16).cuda()
    drop = ops.Dropout(0.1, 3)
    pre, pre16 = ops.Packed8.empty(m, n), torch.empty((m, n), dtype=BF16, device="cuda")
    want = ops.linear(x, w, b, act="silu", dropout=drop, residual=r, pre=pre16)
    got = ops.linear(x, w, b, act="silu", dropout=drop, residual=r, pre=pre)
    assert torch.equal(got, want)
    # against the 16-bit pre: half a step of either rounding
    back = ops.unpack8(pre, torch.float32).double()
    scale = torch.exp2(pre.scales.double() - 127).repeat_interleave(32, 1)[:, :n]
    assert bool(((back - pre16.double()).abs() <= (2.0 ** -4 + 2.0 ** -7) * pre16.double().abs() + 2.0 ** -10 * scale).all())


def test_one_of_x_and_pre_kept():
    g = torch.Generator().manual_seed(4)
    x, w, dy = (torch.randn(s, generator=g).to(BF16).cuda() for s in ((90, 64), (100, 64), (90, 100)))
    pre16 = torch.randn((90, 100), generator=g).to(BF16).cuda()
    x8, pre8 = ops.pack8(x), ops.pack8(pre16)
    xs, ps = ops.unpack8(x8), ops.unpack8(pre8)
    for a, b in ((x8, ps), (xs, pre8), (x8, pre8)):
        want = ops.linear_backward(dy, xs, w, act="gelu", pre=ps)
        got = ops.linear_backward(dy, a, w, act="gelu", pre=b)
        assert all(torch.equal(u, v) for u, v in zip(want, got))
    dx, none, db = ops.linear_backward(dy, x8, w, act="gelu", pre=pre8, need_dw=False)
    assert none is None and torch.equal(dx, want[0]) and torch.equal(db, want[2])
    none, dw, _ = ops.linear_backward(dy, x8, w, act="gelu", pre=pre8, need_dx=False, bias=False)
    assert none is None and torch.equal(dw, want[1])


@pytest.mark.parametrize("dtype", (BF16, F16))
@pytest.mark.parametrize("m,n,k", [(1, 33, 7), (45, 8, 1), (700, 1030, 803), (2300, 40, 2056), ((1 << 20) + 70, 9, 61)])
def test_gradients_have_the_bits_of_values_unpacked_before(m, n, k, dtype):
    """x restored beside the gradient of the activation or apart, w copied or read in
    place, sums of dy alone: the values and so the products are those of the call on
    unpacked arrays."""
    g = torch.Generator(device="cuda").manual_seed(m)
    normal = lambda *s: torch.randn(s, generator=g, device="cuda").to(dtype)  # noqa: E731
    x8, pre8, w, dy = ops.pack8(normal(m, k)), ops.pack8(normal(m, n)), normal(n, k), normal(m, n)
    xs, ps = ops.unpack8(x8, dtype), ops.unpack8(pre8, dtype)
    for act, x_act, drop in (("silu", "none", None), ("gelu", "relu", ops.Dropout(0.2, 9, offset=2, row0=1)), ("none", "relu", None)):
        x = torch.relu(xs) if x_act == "relu" else xs
        kw = {"act": act, "dropout": drop}
        want = ops.linear_backward(dy, x, w, pre=ps if act != "none" else None, **kw)
        for pre in ((ps, pre8) if act != "none" else (None,)):
            got = ops.linear_backward(dy, x8, w, x_act=x_act, pre=pre, **kw)
            assert all(torch.equal(a, b) for a, b in zip(want, got)), (act, x_act)


def test_values_kept_as_nan_and_zeros():
    """A NaN kept in x or pre reaches the sums that hold it, and no others."""
    g = torch.Generator().manual_seed(6)
    z, pre, w, dy = (torch.randn(s, generator=g).to(BF16) for s in ((40, 64), (40, 32), (32, 64), (40, 32)))
    z[3, 5], pre[7, 9] = float("inf"), float("nan")
    dx, dw, db = ops.linear_backward(dy.cuda(), ops.pack8(z.cuda()), w.cuda(), act="silu", pre=ops.pack8(pre.cuda()))
    bad = torch.zeros((32, 64), dtype=torch.bool)
    bad[:, 5], bad[9] = True, True
    assert torch.equal(dw.cpu().isnan(), bad)
    assert dx.cpu().isnan().any(1).nonzero().flatten().tolist() == [7]
    assert db.cpu().isnan().nonzero().flatten().tolist() == [9]


@pytest.mark.parametrize("m,n,k", [(40, 100, 64), (300, 520, 264), (64, 100, 4096), (2100, 2080, 64), (4100, 2200, 256)])
def test_sums_that_are_not_finite_stay_alone(m, n, k):
    """Columns with an infinite or NaN bias, and a row of NaN, in tiles of every size,
    whole and split: NaN there, and the scales of the 32 columns go by the others."""
    g = torch.Generator().manual_seed(n)
    x, w, b = ((torch.randn(s, generator=g) * c).to(BF16) for s, c in (((m, k), 1.0), ((n, k), k ** -0.5), ((n,), 0.5)))
    off = b.clone()
    off[5], off[37], off[n - 1] = float("inf"), float("-inf"), float("nan")
    off[40:45] = float("nan")
    x[m // 2, 3] = float("nan")
    pre = ops.Packed8.empty(m, n)
    y = ops.linear(x.cuda(), w.cuda(), off.cuda(), act="silu", pre=pre)
    bad = ~torch.isfinite(off)[None, :].expand(m, n).clone()
    bad[m // 2] = True
    got = unpack(pre.values, pre.scales)
    assert torch.equal(got.isnan(), bad)
    x[m // 2] = 0
    ref = Linear(x, w, b, None, "silu", None)
    rows = torch.arange(m) != m // 2
    # a finite stand-in for the bad columns that no scale goes by
    q = pre.values.cpu().float()
    q[bad] = 0
    z, bound = torch.where(bad, 0.0, ref.z), torch.where(bad, 0.0, ref.z_bound)
    assert_kept(q[rows].to(F8), pre.scales.cpu()[rows], z[rows], bound[rows], "pre")
    assert bool((pre.scales.cpu()[m // 2] == 1).all())
    assert torch.isfinite(y.cpu()[rows][:, torch.isfinite(off)]).all()


def test_empty():
    w = torch.ones((40, 0), dtype=BF16, device="cuda")
    pre = ops.Packed8.empty(6, 40)
    y = ops.linear(torch.ones((6, 0), dtype=BF16, device="cuda"), w, torch.full((40,), 2.0, dtype=BF16, device="cuda"),
                   act="relu", pre=pre)
    assert bool((y == 2).all()) and bool((ops.unpack8(pre) == 2).all())
    x8 = ops.Packed8.empty(0, 24)
    w = torch.ones((40, 24), dtype=BF16, device="cuda")
    dx, dw, db = ops.linear_backward(torch.ones((0, 40), dtype=BF16, device="cuda"), x8, w, act="gelu",
                                     pre=ops.Packed8.empty(0, 40))
    assert dx.shape == (0, 24) and not dw.any() and not db.any()


def test_refusals():
    x, w, dy = (torch.zeros(s, dtype=BF16, device="cuda") for s in ((8, 16), (24, 16), (8, 24)))
    x8, pre = ops.pack8(x), ops.pack8(dy)
    for call in (lambda: ops.linear(x, w, act="gelu", pre=x8), lambda: ops.linear_backward(dy, x, w, x_act="gelu"),
                 lambda: ops.linear_backward(dy, pre, w), lambda: ops.linear_backward(dy, x8, w, act="gelu"),
                 lambda: ops.linear_backward(dy, x8, w, act="gelu", pre=x8),
                 lambda: ops.linear_backward(dy, x8, w, x_act="tanh")):
        with pytest.raises(ValueError):
            call()
    with pytest.raises(Exception, match="dip_linear_kept"):
        ops.linear(x.float(), w.float(), pre=pre)


def test_graph_and_stream():
    g = torch.Generator().manual_seed(8)
    x, w, dy = (torch.randn(s, generator=g).to(BF16).cuda() for s in ((300, 515), (264, 515), (300, 264)))

    def step(stream=None):
        pre = ops.Packed8.empty(300, 264)
        y = ops.linear(x, w, act="gelu", pre=pre, stream=stream)
        x8 = ops.pack8(x, stream=stream)
        return (y, *ops.linear_backward(dy, x8, w, act="gelu", pre=pre, stream=stream))

    step()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step()
    for _ in range(3):
        x.normal_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(step(), out))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = step(side)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(step(), got))

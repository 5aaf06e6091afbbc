"""dip_rms_norm and dip_rms_norm_grad against their plain 64-bit form, element by
element, within bounds derived from the formats."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from kept_reference import F8, RmsNorm, assert_kept  # noqa: E402
from ops_reference import assert_close  # noqa: E402

if torch.cuda.is_available():
    from paper_2504_14145_amd import ops

F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
TYPES = [F32, BF16, F16]


@pytest.fixture(autouse=True)
def need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


def dev(t):
    return None if t is None else t.cuda()


def put(t, pad, shift):
    """The same values on the GPU in rows of a wider array whose other values are NaN."""
    if t is None or not (pad or shift):
        return dev(t)
    m, c = t.shape
    flat = torch.full((shift + m * (c + pad),), float("nan"), dtype=t.dtype, device="cuda")
    v = flat[shift:].view(m, c + pad)[:, :c]
    v.copy_(t)
    return v


def check(m, c, dtype, residual=True, gamma=True, packed=True, along=True, eps=1e-5, pad=0, shift=0, seed=1, scale=1.0):
    g = torch.Generator().manual_seed(seed)
    normal = lambda *s: torch.randn(s, generator=g)  # noqa: E731
    x = (normal(m, c) * (1 + 5 * torch.rand(c, generator=g) ** 4) * scale).to(dtype)
    r = (normal(m, c) * 2 * scale).to(dtype) if residual else None
    w = (1 + 0.3 * normal(c)).to(dtype) if gamma else None
    dy, dt = (0.3 * normal(m, c)).to(dtype), (normal(m, c)).to(dtype) if along else None
    ref = RmsNorm(x, r, w, eps)
    what = f"{m} x {c} {dtype}"
    out = torch.full((m, c + pad), 7.0, dtype=dtype, device="cuda")
    q8 = torch.full((m, c + pad), 0x5a, dtype=torch.uint8, device="cuda")
    s8 = torch.full((m, (c + 31) // 32 + pad), 0x5b, dtype=torch.uint8, device="cuda")
    p = ops.Packed8(q8.view(F8)[:, :c], s8[:, :(c + 31) // 32]) if packed else None
    y, total, rstd, kept = ops.rms_norm(put(x, pad, shift), dev(w), eps, residual=put(r, pad, shift), packed=p,
                                        out=out[:, :c])
    assert kept is p
    assert torch.equal(total.cpu(), ref.total), what + " total"
    assert_close(rstd, ref.rstd, ref.rel * ref.rstd, F32, what + " rstd")
    assert_close(y, ref.y, ref.y_bound, dtype, what + " y")
    assert bool((out[:, c:] == 7.0).all()) and bool((q8[:, c:] == 0x5a).all()) and bool((s8[:, (c + 31) // 32:] == 0x5b).all())
    if packed:
        assert_kept(p.values, p.scales, ref.y, ref.y_bound, what + " packed")
    dx = torch.full((m, c + pad), 7.0, dtype=dtype, device="cuda")
    _, dg = ops.rms_norm_backward(put(dy, pad, shift), put(total.cpu(), pad, shift), rstd, dev(w), dtotal=put(dt, pad, shift),
                                  dx=dx[:, :c])
    want = ref.grads(dy, dt)
    assert_close(dx[:, :c], *want["dx"], dtype, what + " dx")
    assert bool((dx[:, c:] == 7.0).all())
    if gamma:
        assert_close(dg, *want["dgamma"], dtype, what + " dgamma")
    else:
        assert dg is None


# every number of lanes and vectors a row, its edges, and rows beyond the registers
COLS = (1, 7, 8, 16, 31, 33, 64, 65, 120, 129, 255, 257, 512, 515, 1024, 1027, 2048, 2051, 4096, 4099, 8192, 8195, 16384, 16390,
        40000)


@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("c", COLS)
def test_columns(c, dtype):
    check(5 if c > 2000 else 37, c, dtype, seed=c)


@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("m,c", [(1, 4096), (2, 16), (3000, 40), (1500, 264), (1201, 1795), (700, 4096), (40, 20000)])
def test_rows(m, c, dtype):
    check(m, c, dtype, seed=m)


@pytest.mark.parametrize("residual", [False, True])
@pytest.mark.parametrize("gamma", [False, True])
@pytest.mark.parametrize("packed", [False, True])
def test_options(residual, gamma, packed):
    for c in (100, 1000, 3000, 20000):
        check(9, c, BF16, residual=residual, gamma=gamma, packed=packed, along=packed, seed=c)


@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("pad,shift", [(1, 0), (5, 3), (8, 1), (16, 8)])
def test_strides_and_alignment(dtype, pad, shift):
    for c in (12, 250, 700, 2500, 17000):
        check(6, c, dtype, pad=pad, shift=shift, seed=c)


@pytest.mark.parametrize("eps,scale", [(1e-6, 1e-3), (1e-2, 1.0), (0.0, 1.0), (1e-5, 200.0)])
def test_eps_and_scales(eps, scale):
    check(20, 320, F32, eps=eps, scale=scale)
    check(20, 320, BF16, eps=eps, scale=scale)


@pytest.mark.parametrize("c", [40, 3000, 20000])
def test_total_in_the_residuals_place_and_dx_in_dtotals(c):
    g = torch.Generator().manual_seed(3)
    x, r, dy, dt = (torch.randn((11, c), generator=g).to(BF16).cuda() for _ in range(4))
    w = torch.rand(c, generator=g).to(BF16).cuda()
    want = ops.rms_norm(x, w, residual=r, packed=True)
    grads = ops.rms_norm_backward(dy, want[1], want[2], w, dtotal=dt)
    got = ops.rms_norm(x, w, residual=r, total=r, packed=True)
    assert got[1] is r
    for a, b in zip(want[:3], got[:3]):
        assert torch.equal(a, b)
    assert torch.equal(want[3].values.view(torch.uint8), got[3].values.view(torch.uint8))
    dx, dg = ops.rms_norm_backward(dy, r, got[2], w, dtotal=dt, dx=dt)
    assert dx is dt and torch.equal(dx, grads[0]) and torch.equal(dg, grads[1])


@pytest.mark.parametrize("c", [48, 1500, 20000])
def test_outputs_that_are_not_wanted(c):
    g = torch.Generator().manual_seed(4)
    x, dy = (torch.randn((65, c), generator=g).to(F16).cuda() for _ in range(2))
    w = torch.rand(c, generator=g).to(F16).cuda()
    y, total, rstd, p = ops.rms_norm(x, w, packed=True)
    assert total is x
    y2, _, rstd2, p2 = ops.rms_norm(x, w, packed=True, need_out=False)
    assert y2 is None and torch.equal(rstd, rstd2) and torch.equal(p.scales, p2.scales)
    assert torch.equal(p.values.view(torch.uint8), p2.values.view(torch.uint8))
    dx, dg = ops.rms_norm_backward(dy, x, rstd, w)
    a, none = ops.rms_norm_backward(dy, x, rstd, w, need_dgamma=False)
    assert none is None and torch.equal(a, dx)
    none, b = ops.rms_norm_backward(dy, x, rstd, w, need_dx=False)
    assert none is None and torch.equal(b, dg)
    assert ops.rms_norm_backward(dy, x, rstd, w, need_dx=False, need_dgamma=False) == (None, None)


@pytest.mark.parametrize("c", [48, 3000, 20000])
def test_accumulated_gradients(c):
    """Two pieces of a sample add up in float32 to what the whole gives."""
    g = torch.Generator().manual_seed(5)
    x, dy = (torch.randn((90, c), generator=g).to(BF16) for _ in range(2))
    w = torch.rand(c, generator=g).to(BF16)
    ref = RmsNorm(x, None, w, 1e-5)
    acc = torch.full((c,), 0.5, device="cuda")
    for a, b in ((0, 31), (31, 90)):
        _, total, rstd, _ = ops.rms_norm(x[a:b].cuda(), w.cuda())
        _, got = ops.rms_norm_backward(dy[a:b].cuda(), total, rstd, w.cuda(), dgamma=acc, accumulate=True)
        assert got is acc
    want, bound = ref.grads(dy, None)["dgamma"]
    assert_close(acc, want + 0.5, bound + 4 * 2.0 ** -24 * (want.abs() + 0.5), F32, "dgamma")


def test_gradient_against_differences():
    g = torch.Generator().manual_seed(6)
    x, dy, dt = (torch.randn((3, 70), generator=g) for _ in range(3))
    w = torch.rand(70, generator=g) + 0.5
    _, total, rstd, _ = ops.rms_norm(x.cuda(), w.cuda())
    dx, dg = ops.rms_norm_backward(dy.cuda(), total, rstd, w.cuda(), dtotal=dt.cuda())

    def loss(x, w):
        ref = RmsNorm(torch.zeros((3, 70)), None, None, 1e-5)
        ref.__dict__.update(total=x)
        y = x / torch.sqrt((x * x).mean(1, keepdim=True) + 1e-5) * w
        return float((y * dy.double()).sum() + (x * dt.double()).sum())

    x64, w64, h = x.double(), w.double(), 1e-5
    for i, j in ((0, 0), (1, 33), (2, 69)):
        d = torch.zeros_like(x64)
        d[i, j] = h
        # central differences: h^2 of the third derivative and 2^-52 / h of the loss, below 1e-8
        assert abs((loss(x64 + d, w64) - loss(x64 - d, w64)) / (2 * h) - float(dx[i, j])) < 1e-5
        d = torch.zeros_like(w64)
        d[j] = h
        assert abs((loss(x64, w64 + d) - loss(x64, w64 - d)) / (2 * h) - float(dg[j])) < 1e-5


def test_values_that_are_not_finite_stay_in_their_row():
    x = torch.ones((4, 96), dtype=BF16)
    x[1, 5], x[2, 7] = float("inf"), float("nan")
    y, _, rstd, p = ops.rms_norm(x.cuda(), packed=True)
    y, back = y.cpu().float(), ops.unpack8(p).cpu().float()
    assert bool((y[[0, 3]] - 1).abs().max() < 1e-2) and bool((back[[0, 3]] - 1).abs().max() < 0.07)
    assert float(rstd[1]) == 0 and bool(y[1, 5].isnan()) and bool((y[1, 6:] == 0).all()) and bool(y[2].isnan().all())
    assert bool(back[2].isnan().all()) and bool(back[1, 5].isnan())


def test_empty():
    y, total, rstd, p = ops.rms_norm(torch.zeros((0, 8), device="cuda"), packed=True)
    assert y.shape == (0, 8) and rstd.shape == (0,) and p.shape == (0, 8)
    y, _, rstd, _ = ops.rms_norm(torch.zeros((3, 0), device="cuda"), eps=0.25)
    assert y.shape == (3, 0) and rstd.tolist() == [2.0, 2.0, 2.0]
    w = torch.ones(8, device="cuda")
    dx, dg = ops.rms_norm_backward(torch.zeros((0, 8), device="cuda"), torch.zeros((0, 8), device="cuda"),
                                   torch.zeros(0, device="cuda"), w)
    assert dx.shape == (0, 8) and dg.tolist() == [0.0] * 8
    acc = torch.full((8,), 3.0, device="cuda")
    ops.rms_norm_backward(torch.zeros((0, 8), device="cuda"), torch.zeros((0, 8), device="cuda"),
                          torch.zeros(0, device="cuda"), w, dgamma=acc, accumulate=True)
    assert acc.tolist() == [3.0] * 8


def test_refusals():
    x, w = torch.zeros((4, 40), device="cuda"), torch.zeros(40, device="cuda")
    r = torch.zeros(4, device="cuda")
    for call in (lambda: ops.rms_norm(x[0]), lambda: ops.rms_norm(x, w[:39]), lambda: ops.rms_norm(x, w.half()),
                 lambda: ops.rms_norm(x, residual=x[:3]), lambda: ops.rms_norm(x, total=x.clone()),
                 lambda: ops.rms_norm(x, packed=ops.Packed8.empty(4, 41)), lambda: ops.rms_norm(x, rstd=r[:3]),
                 lambda: ops.rms_norm(x.T), lambda: ops.rms_norm_backward(x, x, None),
                 lambda: ops.rms_norm_backward(x, x, r.double()), lambda: ops.rms_norm_backward(x, x, r, dgamma=w),
                 lambda: ops.rms_norm_backward(x, x, r, w, accumulate=True),
                 lambda: ops.rms_norm_backward(x, x, r, w, dtotal=x.half())):
        with pytest.raises(ValueError):
            call()


def test_forward_of_recorded_tensors_warns():
    x = torch.zeros((4, 40), device="cuda", requires_grad=True)
    with pytest.warns(UserWarning, match="rms_norm records no gradients"):
        ops.rms_norm(x)
    with pytest.warns(UserWarning, match="pack8 records no gradients"):
        ops.pack8(x)


def test_graph_and_stream():
    g = torch.Generator().manual_seed(7)
    x, r, dy = (torch.randn((300, 2056), generator=g).to(BF16).cuda() for _ in range(3))
    w = torch.rand(2056, generator=g).to(BF16).cuda()
    acc = torch.zeros(2056, device="cuda")

    def step(stream=None):
        y, total, rstd, p = ops.rms_norm(x, w, residual=r, packed=True, stream=stream)
        dx, dg = ops.rms_norm_backward(dy, total, rstd, w, dtotal=dy, stream=stream)
        return y, total, rstd, ops.unpack8(p, stream=stream), dx, dg

    step()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step()
        ops.rms_norm_backward(dy, out[1], out[2], w, need_dx=False, dgamma=acc, accumulate=True)
    acc.zero_()
    for i in range(3):
        x.normal_()
        before = acc.clone()
        graph.replay()
        torch.cuda.synchronize()
        want = step()
        for a, b in zip(want, out):
            assert torch.equal(a, b)
        ops.rms_norm_backward(dy, want[1], want[2], w, need_dx=False, dgamma=before, accumulate=True)
        assert torch.equal(before, acc)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = step(side)
    side.synchronize()
    for a, b in zip(step(), got):
        assert torch.equal(a, b)

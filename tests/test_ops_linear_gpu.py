"""dip_linear and dip_linear_grad against their plain 64-bit form, element by
element, within bounds derived from the formats."""
import itertools

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from ops_reference import Linear, assert_close, mask  # noqa: E402

if torch.cuda.is_available():
    import paper_2504_14145_amd as dip
    from paper_2504_14145_amd import ops

BF16, F16 = torch.bfloat16, torch.float16
ACTS = ("none", "relu", "silu", "gelu")


@pytest.fixture(autouse=True)
def need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


def normal(gen, shape, dtype, scale=1.0):
    return (torch.randn(shape, generator=gen) * scale).to(dtype)


def strided(t, pad, shift=0):
    """The same values on the GPU in rows of a wider array, `shift` elements into
    an allocation whose other values are NaN."""
    rows, cols = t.shape
    ld = cols + pad
    flat = torch.full((shift + rows * ld + 8,), float("nan"), dtype=t.dtype, device="cuda")
    v = flat[shift:shift + rows * ld].view(rows, ld)[:, :cols]
    v.copy_(t)
    return v


def inputs(m, n, k, dtype, bias, residual, p, seed):
    g = torch.Generator().manual_seed(seed)
    x, w = normal(g, (m, k), dtype), normal(g, (n, k), dtype, max(k, 1) ** -0.5)
    b = normal(g, (n,), dtype, 0.5) if bias else None
    r = normal(g, (m, n), dtype) if residual else None
    drop = ops.Dropout(p, seed * 77 + 5, offset=seed, row0=seed % 1000) if p else None
    return x, w, b, r, drop, normal(g, (m, n), dtype, 0.3)


def dev(t):
    return None if t is None else t.cuda()


def check(m, n, k, dtype, act="none", bias=True, residual=False, p=0.0, seed=1, pads=(0, 0),
          shift=0, backward=True):
    x, w, b, r, drop, dy = inputs(m, n, k, dtype, bias, residual, p, seed)
    ref = Linear(x, w, b, r, act, drop)
    put = (lambda t: strided(t, pads[0], shift)) if pads[0] or shift else dev
    gx, gw, gdy = put(x), put(w), put(dy)
    gr = None if r is None else put(r)
    pre = torch.full((m, n + pads[1]), float("nan"), dtype=dtype, device="cuda")[:, :n]
    out = torch.full((m, n + pads[1]), 7.0, dtype=dtype, device="cuda")
    y = ops.linear(gx, gw, dev(b), act=act, dropout=drop, residual=gr, pre=pre, out=out[:, :n])
    what = f"m {m} n {n} k {k} {dtype} {act} p {p}"
    assert_close(pre, ref.z, ref.z_bound, dtype, what + " pre")
    assert_close(y, ref.y, ref.y_bound, dtype, what + " y")
    assert bool((out[:, n:] == 7.0).all()), "columns beyond n were written"
    if not backward:
        return
    dx = torch.full((m, k + pads[1]), 7.0, dtype=dtype, device="cuda")
    dw = torch.full((n, k + pads[1]), 7.0, dtype=dtype, device="cuda")
    _, _, db = ops.linear_backward(gdy, gx, gw, act=act, dropout=drop, pre=pre if act != "none" else None,
                                   bias=True, dx=dx[:, :k], dw=dw[:, :k])
    want = ref.grads(dy, pre if act != "none" else None, dtype)
    for name, got in (("dx", dx[:, :k]), ("dw", dw[:, :k]), ("db", db)):
        assert_close(got, *want[name], dtype, f"{what} {name}")
    assert bool((dx[:, k:] == 7.0).all()) and bool((dw[:, k:] == 7.0).all())


@pytest.mark.parametrize("dtype", [BF16, F16], ids=str)
@pytest.mark.parametrize("m,n,k", [(1, 1, 1), (1, 64, 64), (2, 8, 2048), (5, 100, 72), (16, 136, 1024),
                                   (17, 33, 65), (64, 256, 96), (65, 130, 200), (128, 128, 128),
                                   (129, 257, 40), (255, 72, 511), (300, 520, 264)])
def test_shapes(m, n, k, dtype):
    check(m, n, k, dtype, act=ACTS[(m + n + k) % 4], residual=bool(m % 2), seed=m)


@pytest.mark.parametrize("act,bias,residual,p", itertools.product(ACTS, (False, True), (False, True), (0.0, 0.3)))
def test_epilogues(act, bias, residual, p):
    check(70, 90, 48, BF16, act=act, bias=bias, residual=residual, p=p, seed=3)


@pytest.mark.parametrize("pads,shift", [((8, 8), 0), ((8, 0), 8), ((3, 5), 0), ((8, 1), 1), ((0, 0), 1),
                                        ((1, 0), 4), ((16, 24), 16)])
@pytest.mark.parametrize("m,n,k", [(37, 48, 64), (130, 150, 77), (1, 40, 264)])
def test_strides_and_alignment(m, n, k, pads, shift):
    check(m, n, k, F16, act="gelu", residual=True, p=0.25, seed=9, pads=pads, shift=shift)


@pytest.mark.parametrize("m,n,k", [(513, 384, 1100), (260, 2100, 320), (1030, 70, 130), (96, 1024, 2048),
                                   (33, 4100, 520)])
def test_larger(m, n, k):
    check(m, n, k, BF16, act="silu", seed=m)


def test_long_contraction():
    """Few outputs over a long axis, forward and the weight's gradient."""
    check(40, 48, 16384, BF16, seed=2, backward=False)
    check(20000, 24, 40, BF16, act="none", seed=4)


@pytest.mark.parametrize("m,n,k", [(0, 16, 16), (16, 0, 16), (7, 24, 0)])
def test_sizes_of_zero(m, n, k):
    dtype = BF16
    x, w, b, r, drop, dy = inputs(m, n, k, dtype, True, True, 0.2, 3)
    y = ops.linear(dev(x), dev(w), dev(b), act="silu", dropout=drop, residual=dev(r))
    ref = Linear(x, w, b, r, "silu", drop)
    assert_close(y, ref.y, ref.y_bound, dtype, "y")
    pre = torch.zeros((m, n), dtype=dtype, device="cuda")
    dx, dw, db = ops.linear_backward(dev(dy), dev(x), dev(w), act="silu", dropout=drop, pre=pre)
    want = ref.grads(dy, pre, dtype)
    for name, got in (("dx", dx), ("dw", dw), ("db", db)):
        assert_close(got, *want[name], dtype, name)


@pytest.mark.parametrize("m,n,k", [(50, 70, 90), (256, 512, 64)])
def test_gradients_accumulate_in_float32(m, n, k):
    x, w, b, r, drop, dy = inputs(m, n, k, BF16, True, False, 0.1, 5)
    ref = Linear(x, w, b, r, "none", drop)
    dw = torch.full((n, k), 2.0, device="cuda")
    db = torch.full((n,), -1.0, device="cuda")
    for _ in range(2):
        ops.linear_backward(dev(dy), dev(x), dev(w), dropout=drop, dw=dw, db=db, accumulate=True, need_dx=False)
    want = ref.grads(dy, None, BF16)
    for got, name, start in ((dw, "dw", 2.0), (db, "db", -1.0)):
        v, bound = want[name]
        total = start + 2 * v
        assert_close(got, total, 2 * bound + 8 * 2.0 ** -24 * (abs(start) + 2 * v.abs()), torch.float32, name)


def test_gradients_one_by_one():
    x, w, b, r, drop, dy = inputs(90, 60, 30, F16, True, False, 0.0, 6)
    args = dev(dy), dev(x), dev(w)
    whole = ops.linear_backward(*args)
    for i, need in enumerate((dict(need_dw=False, bias=False), dict(need_dx=False, bias=False),
                              dict(need_dx=False, need_dw=False))):
        got = ops.linear_backward(*args, **need)
        assert [t is None for t in got] == [j != i for j in range(3)]
        assert torch.equal(got[i], whole[i])


def test_gradient_against_differences():
    """Directional differences of the 64-bit forward against the kernel's gradients."""
    m, n, k, act = 40, 56, 64, "gelu"
    x, w, b, r, drop, dy = inputs(m, n, k, F16, True, True, 0.2, 8)
    keep = mask(drop, m, n)
    pre = torch.empty((m, n), dtype=F16, device="cuda")
    ops.linear(dev(x), dev(w), dev(b), act=act, dropout=drop, residual=dev(r), pre=pre)
    grads = ops.linear_backward(dev(dy), dev(x), dev(w), act=act, dropout=drop, pre=pre)
    g = torch.Generator().manual_seed(1)
    base = [x.double(), w.double(), b.double()]
    for i, grad in enumerate(grads):
        d = torch.randn(base[i].shape, generator=g).double()
        loss = []
        for h in (1e-5, -1e-5):
            at = [v + h * d if j == i else v for j, v in enumerate(base)]
            loss.append((Linear(*at, r, act, drop, keep).y * dy.double()).sum())
        want = float((loss[0] - loss[1]) / 2e-5)
        got = float((grad.cpu().double() * d).sum())
        # pre, g and the gradient are each rounded to 11 bits, their errors
        # independent from element to element; differences are good to 1e-9
        size = float((grad.cpu().double().abs() * d.abs()).norm())
        assert abs(got - want) <= 6 * 3 * 2.0 ** -11 * size + 1e-6 * abs(want), (i, got, want)


def test_infinities_under_the_mask_are_gone():
    m, n, k = 33, 80, 40
    x, w, b, r, drop, dy = inputs(m, n, k, BF16, True, True, 0.5, 4)
    keep = mask(drop, m, n)
    w[3] = float("inf")          # column 3 of the product is NaN or infinite
    dy[:, 3] = float("nan")
    dy[:, 5] = float("inf")
    y = ops.linear(dev(x), dev(w), dev(b), dropout=drop, residual=dev(r)).cpu()
    assert torch.equal(y[~keep], r[~keep])
    _, _, db = ops.linear_backward(dev(dy), dev(x), dev(w), dropout=drop)
    g = torch.where(keep, dy.float() * drop.scale, torch.tensor(0.0)).sum(0)
    assert torch.equal(torch.isnan(db.cpu()), torch.isnan(g)) and torch.equal(torch.isinf(db.cpu()), torch.isinf(g))


def test_a_piece_draws_its_samples_mask():
    """Rows 20.. as a piece of their own, with row0 advanced, equal the whole's."""
    x, w, b, r, _, _ = inputs(48, 72, 32, BF16, True, True, 0.0, 4)
    whole = ops.linear(dev(x), dev(w), dev(b), dropout=ops.Dropout(0.4, 11, 2), residual=dev(r))
    piece = ops.linear(dev(x[20:]), dev(w), dev(b), dropout=ops.Dropout(0.4, 11, 2, row0=20), residual=dev(r[20:]))
    assert torch.equal(whole[20:], piece)


def test_the_result_may_replace_the_residual():
    x, w, b, r, drop, _ = inputs(130, 260, 64, BF16, True, True, 0.1, 4)
    want = ops.linear(dev(x), dev(w), dev(b), dropout=drop, residual=dev(r))
    both = dev(r)
    ops.linear(dev(x), dev(w), dev(b), dropout=drop, residual=both, out=both)
    assert torch.equal(want, both)


def test_same_call_same_bits_on_another_stream_and_in_a_graph():
    m, n, k = 200, 300, 520
    x, w, b, r, drop, dy = (dev(t) if isinstance(t, torch.Tensor) else t
                            for t in inputs(m, n, k, BF16, True, True, 0.1, 4))

    def step(stream=None, pre=None, y=None, **grads):
        pre = torch.empty((m, n), dtype=BF16, device="cuda") if pre is None else pre
        y = ops.linear(x, w, b, act="gelu", dropout=drop, residual=r, pre=pre, out=y, stream=stream)
        return (y, *ops.linear_backward(dy, x, w, act="gelu", dropout=drop, pre=pre, stream=stream, **grads))

    want = step()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = step(side)
    side.synchronize()
    assert all(torch.equal(a, c) for a, c in zip(want, got))
    with torch.cuda.stream(side):
        step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = step()
    for _ in range(3):
        for t in held:
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, c) for a, c in zip(want, held))
        again = step()
        assert all(torch.equal(a, c) for a, c in zip(want, again))


def test_refusals():
    x, w, b, r, drop, dy = inputs(8, 16, 24, BF16, True, True, 0.1, 1)
    x, w, b, r, dy = (t.cuda() for t in (x, w, b, r, dy))
    with pytest.raises(ValueError):
        ops.linear(x, w.to(F16))
    with pytest.raises(ValueError):
        ops.linear(x, w[:, :20])
    with pytest.raises(ValueError):
        ops.linear(x.cpu(), w)
    with pytest.raises(ValueError):
        ops.linear(x, w, b[:8])
    with pytest.raises(ValueError):
        ops.linear(x, w, act="tanh")
    with pytest.raises(ValueError):
        ops.linear(x.t().contiguous().t(), w)
    with pytest.raises(ValueError):
        ops.linear(x, w, residual=r[:4])
    with pytest.raises(ValueError):
        ops.Dropout(1.0, 1)
    with pytest.raises(ValueError):
        ops.linear_backward(dy, x, w, act="gelu")
    with pytest.raises(ValueError):
        ops.linear_backward(dy, x, w, accumulate=True)
    with pytest.raises(ValueError):
        ops.linear_backward(dy, x, w, dw=torch.empty((16, 24), device="cuda"), db=torch.empty(16, dtype=BF16, device="cuda"))
    with pytest.raises(dip.DipSimError) as e:
        ops.linear(x.float(), w.float())
    assert e.value.code == dip.E_UNSUPPORTED
    with pytest.raises(dip.DipSimError) as e:
        ops.linear(x, w, dropout=ops.Dropout(0.5, 1, row0=(1 << 32) - 4))
    assert e.value.code == dip.E_RANGE

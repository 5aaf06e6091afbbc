"""dip_rms_norm to the last bit: the statistics of a row are those of 64 bits, and y is
rounded once.

Squares are exact in float64 and a thread adds at most 8 ceil(c / 8192) of them, so rstd
before its rounding is within 2^-41 of the value; half a step of float32 is 2^-24."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

if torch.cuda.is_available():
    from paper_2504_14145_amd import ops

F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
TYPES = [F32, BF16, F16]
STEP = 2.0 ** -24 * (1 + 2.0 ** -10)


@pytest.fixture(autouse=True)
def need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


def rows(c, dtype, seed):
    """Rows whose sums of squares lose most where they are summed in 32 bits: equal
    values, one that stands above the others, many small ones behind a large one."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.randn((8, c), generator=g, device="cuda")
    x[0], x[1], x[2] = 0.1, 1 + 2.0 ** -7, 3.3
    x[3] = 1e-2
    x[3, c // 3] = 57.3
    x[4, : c // 2], x[4, c // 2:] = 1.3, -0.9
    x[5] = torch.linspace(0.5, 2.0, c, device="cuda")
    return x.to(dtype)


def statistics(x, eps):
    d = x.double()
    return 1 / torch.sqrt((d * d).sum(1) / x.shape[1] + float(torch.tensor(eps)))   # eps is a float32


@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("c", [1, 24, 64, 100, 250, 510, 700, 1024, 3001, 8192, 8200, 16384, 16390, 100000, 1 << 22])
def test_statistics_are_those_of_64_bits(c, dtype):
    x = rows(c, dtype, c)
    for eps in (0.0, 1e-5):
        want = statistics(x, eps)
        y, _, rstd, _ = ops.rms_norm(x, eps=eps)
        assert bool(((rstd.double() - want).abs() <= STEP * want).all()), f"{c} {dtype} {eps} rstd"
        v = x.double() * want[:, None]
        step = STEP if dtype is F32 else torch.finfo(dtype).eps / 2 + STEP
        floor = 0.0 if dtype is not F16 else 2.0 ** -25     # half a step of float16 below its normal range
        assert bool(((y.double() - v).abs() <= step * v.abs() + floor).all()), f"{c} {dtype} {eps} y"


@pytest.mark.parametrize("c", [40, 1000, 5000, 20000])
@pytest.mark.parametrize("dtype", [F32, BF16], ids=str)
def test_rows_whose_squares_no_float32_holds(c, dtype):
    """Magnitudes from 2^-60 to 2^100: rstd is a float32 for all of them."""
    for e in (-60, -30, 60, 100):
        x = torch.ldexp(rows(c, F32, c), torch.tensor(e, device="cuda")).to(dtype)
        want = statistics(x, 0.0)
        y, _, rstd, p = ops.rms_norm(x, eps=0.0, packed=True)
        assert bool(((rstd.double() - want).abs() <= STEP * want).all()), f"{c} {dtype} 2^{e}"
        v = x.double() * want[:, None]
        assert bool(((y.double() - v).abs() <= (torch.finfo(dtype).eps / 2 + STEP) * v.abs()).all()), f"{c} {dtype} 2^{e}"
        back = ops.unpack8(p, F32).double()
        scale = torch.exp2(p.scales.double() - 127).repeat_interleave(32, 1)[:, :c]
        assert bool(((back - v).abs() <= (2.0 ** -4 + STEP) * v.abs() + 2.0 ** -10 * scale).all()), f"{c} {dtype} 2^{e} packed"


def to_8_bits(v):
    """(values, scale bytes, distance from the nearest middle of two 8-bit values in their
    steps) of a float64 matrix on the GPU, from the format's definition."""
    m, n = v.shape
    pad = torch.nn.functional.pad(v, (0, -n % 32)).reshape(m, -1, 32)
    most = pad.abs().amax(2)
    e = torch.frexp(most)[1].double() - 1                      # most in [2^e, 2^(e + 1)), 0 of 0
    e = torch.where(most > 1.75 * torch.exp2(e), e - 7, e - 8).clamp_min(-126)
    e = torch.where(most > 0, e, -126.0)
    q = pad * torch.exp2(-e)[:, :, None]
    step = torch.exp2(torch.frexp(q.abs().clamp_min(2.0 ** -6))[1].double() - 4)
    r = q / step
    middle = (r - torch.floor(r) - 0.5).abs()
    back = lambda t: t.reshape(m, -1)[:, :n]  # noqa: E731
    return back(torch.round(r) * step), (e + 127).to(torch.uint8), back(middle)


def check_8_bits(p, v, sure=2.0 ** -40):
    """Bit by bit.  v is off by 2^-49 of itself and at most 16 steps, so the side of what
    is ``sure`` steps or more from a middle is known, and of these inputs every one is."""
    want, scales, middle = to_8_bits(v)
    assert bool((middle > sure).all()) or sure == 0
    assert torch.equal(p.scales, scales)
    got = p.values.float().double()
    assert torch.equal(got, want), f"{int((got != want).sum())} of {got.numel()}"


@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("m,c", [(300, 64), (2000, 510), (900, 1027), (700, 4096), (40, 16384), (30, 20000)])
def test_y_is_rounded_once(m, c, dtype):
    g = torch.Generator(device="cuda").manual_seed(m)
    x = (torch.randn((m, c), generator=g, device="cuda") * 3).to(dtype)
    w = torch.randn(c, generator=g, device="cuda").to(dtype)
    y, _, _, _ = ops.rms_norm(x, w, eps=0.0)
    v = x.double() * statistics(x, 0.0)[:, None] * w.double()
    step = STEP if dtype is F32 else torch.finfo(dtype).eps / 2 + STEP
    floor = 0.0 if dtype is not F16 else 2.0 ** -25
    assert bool(((y.double() - v).abs() <= step * v.abs() + floor).all())


@pytest.mark.parametrize("c", [40, 1000, 3000, 20000])
@pytest.mark.parametrize("dtype", [F32, BF16], ids=str)
def test_gamma_times_a_row_that_float32_does_not_hold(c, dtype):
    """y and the 8 bits are gamma t rstd where gamma t alone would be infinite."""
    x = rows(c, F32, 1).clamp(-8, 8)
    w = torch.linspace(0.5, 1.0, c, device="cuda")
    for to_x, to_w in ((2.0 ** 100, 2.0 ** 40), (2.0 ** 4, 2.0 ** 124), (2.0 ** -90, 2.0 ** 126)):
        xs, ws = (x * to_x).to(dtype), (w * to_w).to(dtype)
        y, _, _, p = ops.rms_norm(xs, ws, eps=0.0, packed=True)
        v = xs.double() * statistics(xs, 0.0)[:, None] * ws.double()
        inside = v.abs() < torch.finfo(dtype).max / 2
        bound = (torch.finfo(dtype).eps / 2 + STEP) * v.abs()
        assert bool(((y.double() - v).abs() <= bound)[inside].all()), (to_x, to_w)
        assert torch.isfinite(p.values.float())[inside].all()


@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("c", [64, 512, 1000, 3584, 10000, 30000])
def test_every_8_bits_are_those_of_the_64_bit_value(c, dtype):
    """Of 2^25 values some sixty have a float32 that lies on the middle of two 8-bit ones,
    beside which the value itself is, and one in 2^19 a scale that it decides."""
    g = torch.Generator(device="cuda").manual_seed(c)
    m = (1 << 25) // c
    x = torch.randn((m, c), generator=g, device="cuda").to(dtype)
    w = (1 + 0.3 * torch.randn(c, generator=g, device="cuda")).to(dtype)
    eps = 2.0 ** -17
    _, _, _, p = ops.rms_norm(x, w, eps=eps, packed=True, need_out=False)
    v = x.double() * statistics(x, eps)[:, None] * w.double()
    check_8_bits(p, v)


def test_middles_and_what_lies_beside_them():
    """Rows whose rstd is 1, or beside it by the rounding of eps, so that y = gamma t:
    middles of 8-bit values go to the even one; products of two float32 a 2^-28th beside a
    middle, which float32 rounds onto it, go to their side."""
    mid = torch.tensor([(2 * i + 1) / 16 * 2.0 ** e for e in (0, 1, 3) for i in range(8, 16)])      # 17/16, 19/16, ..
    n = len(mid)
    near, far = 1 + 2.0 ** -14, 1 - 2.0 ** -14                 # their product is 1 - 2^-28
    for t, w in ((1.0, mid), (near, mid * far), (-near, mid * far), (near, mid * near), (1.0, -mid)):
        for c in (32, 64, 2048, 20000):
            x, gamma = torch.zeros((1, c)), torch.ones(c)
            x[0, :n], x[0, n], gamma[:n], gamma[n] = t, 1.0, w, 448 * 2.0 ** -4     # the scale is 2^-4
            mean = float((x.double() ** 2).sum()) / c
            eps = float(torch.tensor(1 - mean))
            _, _, _, p = ops.rms_norm(x.cuda(), gamma.cuda(), eps=eps, packed=True, need_out=False)
            check_8_bits(p, (x.double() * gamma.double() / (mean + eps) ** 0.5).cuda(), sure=0)


def test_a_largest_value_beside_the_border_of_two_scales():
    """Products that float32 rounds to 448 from either side: the larger ones take the next
    scale."""
    x, g = torch.zeros((1, 96)), torch.ones(96)
    near, far = 1 + 2.0 ** -13, 1 - 2.0 ** -13                 # squares 2^-26 and more beside 1
    for at, t, w in ((0, near, 448 * far), (32, near, 448 * near), (64, 1.0, 448.0)):
        x[0, at], g[at] = t, w
        x[0, at + 1], g[at + 1] = 1.0, 17.0
    mean = float((x.double() ** 2).mean())
    eps = float(torch.tensor(1 - mean))
    _, _, _, p = ops.rms_norm(x.cuda(), g.cuda(), eps=eps, packed=True, need_out=False)
    check_8_bits(p, (x.double() * g.double() / (mean + eps) ** 0.5).cuda(), sure=0)


@pytest.mark.parametrize("c", [40, 1027, 3000, 12345, 20000])
def test_y_in_the_residuals_place(c):
    g = torch.Generator(device="cuda").manual_seed(c)
    x, r = (torch.randn((70, c), generator=g, device="cuda").to(BF16) for _ in range(2))
    w = torch.rand(c, generator=g, device="cuda").to(BF16)
    want = ops.rms_norm(x, w, residual=r, packed=True)
    got = ops.rms_norm(x, w, residual=r, packed=True, out=r)
    assert got[0] is r and all(torch.equal(a, b) for a, b in zip(want[:3], got[:3]))
    assert torch.equal(want[3].values.view(torch.uint8), got[3].values.view(torch.uint8))
    assert torch.equal(want[3].scales, got[3].scales)

"""The conversions to and from 8 bits over all that they take: every 16-bit value under every
scale that it can have, float32 beside every border, every byte under every scale."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from kept_reference import F8  # noqa: E402

if torch.cuda.is_available():
    from paper_2504_14145_amd import ops

F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16


@pytest.fixture(autouse=True)
def need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


def to_nearest(q):
    """float64 values of magnitude up to 448 to four significant bits, steps of at least
    2^-9, ties to even."""
    step = torch.exp2((torch.frexp(q.abs().clamp_min(2.0 ** -6))[1] - 4).double())
    return torch.round(q / step) * step


def check_group(values, e, dtype):
    """Values of magnitude up to 448 2^e, in rows of 32 that begin with a value which has
    the scale 2^e."""
    # the largest there is: 448 2^e itself or, where the type does not hold it (1.75 2^-24 in
    # float16, all but 2^-24 of which is finer than its steps), the next below
    most = float(values.double().abs().max())
    assert most <= 448 * 2.0 ** e and (most > 224 * 2.0 ** e or e == -126)
    x = torch.full(((len(values) + 30) // 31, 32), most, dtype=dtype, device="cuda")
    rest = torch.zeros(x.shape[0] * 31, dtype=dtype, device="cuda")
    rest[:len(values)] = values
    x[:, 1:] = rest.view(-1, 31)
    p = ops.pack8(x)
    assert bool((p.scales == e + 127).all()), e
    want = to_nearest(x.double() * 2.0 ** -e)
    assert torch.equal(p.values.float().double(), want), e
    assert torch.equal(p.values.view(torch.uint8) >= 128, torch.signbit(x)), e


@pytest.mark.parametrize("dtype", [BF16, F16], ids=str)
def test_every_value_under_every_scale(dtype):
    v = torch.arange(1 << 16, device="cuda").to(torch.int32).to(torch.int16).view(dtype)
    v = v[torch.isfinite(v)]
    f = torch.finfo(dtype)
    tiny = f.smallest_normal * f.eps
    for e in range(-126, 128):
        if 448 * 2.0 ** e < tiny or (e > -126 and 448 * 2.0 ** (e - 1) >= f.max):
            continue
        inside = v[v.double().abs() <= min(448 * 2.0 ** e, f.max)]
        check_group(inside, e, dtype)


def test_float32_beside_every_border():
    """The middles of neighbouring 8-bit values and the float32 on either side of them,
    the values themselves, and random ones, under every scale."""
    g = torch.Generator(device="cuda").manual_seed(1)
    q = torch.arange(127, dtype=torch.uint8).view(F8).double()
    mid = (q[1:] + q[:-1]) / 2
    base = torch.cat((q, mid)).cuda()
    for e in range(-126, 120):
        v = (base * 2.0 ** e).float()                           # exact but below float32's normal range
        up = torch.nextafter(v, torch.full_like(v, float("inf")))
        down = torch.nextafter(v, torch.full_like(v, float("-inf")))
        r = (torch.rand(2000, generator=g, device="cuda", dtype=torch.double) * 448 * 2.0 ** e).float()
        r = r * torch.exp2(-20 * torch.rand(2000, generator=g, device="cuda"))
        v = torch.cat((v, up, down, r))
        v = v[v.double().abs() <= min(448 * 2.0 ** e, torch.finfo(F32).max)]
        check_group(torch.cat((v, -v)), e, F32)


@pytest.mark.parametrize("to", [F32, BF16, F16], ids=str)
def test_every_byte_under_every_scale(to):
    """All 256 scales times all 256 values: exact, or rounded once, and what lies beyond
    the type's largest value is that."""
    s = torch.arange(256, device="cuda").to(torch.uint8).repeat_interleave(8).view(256, 8)
    q = torch.arange(256, device="cuda").to(torch.uint8).expand(256, 256).contiguous()
    v = q.view(F8).float().double() * torch.exp2(s.double() - 127).repeat_interleave(32, 1)
    v[255] = float("nan")
    f = torch.finfo(to)
    want = v.clamp(f.min, f.max).to(to)
    got = ops.unpack8(ops.Packed8(q.view(F8), s), to)
    assert torch.equal(got.isnan(), want.isnan())
    assert torch.equal(got.nan_to_num(0), want.nan_to_num(0))


@pytest.mark.parametrize("m,n,k", [(40, 100, 64), (300, 520, 264), (64, 100, 4096), (2000, 1500, 128), (4100, 2200, 64),
                                   (1152, 3840, 64), (5, 70, 256)])
@pytest.mark.parametrize("dtype", [BF16, F16], ids=str)
def test_a_product_keeps_what_packing_its_sums_keeps(m, n, k, dtype):
    """Operands whose products are eighths and whose sums float32 holds exactly in any
    order, in tiles of every size, whole and split: bit by bit what packing them gives."""
    g = torch.Generator(device="cuda").manual_seed(m)
    x = torch.randint(-3, 4, (m, k), generator=g, device="cuda").to(dtype)
    w = (torch.randint(-5, 6, (n, k), generator=g, device="cuda") / 8).to(dtype)
    b = (torch.randint(-400, 400, (n,), generator=g, device="cuda") / 8).to(dtype)
    pre = ops.Packed8.empty(m, n)
    y = ops.linear(x, w, b, act="relu", pre=pre)
    z = x.float() @ w.float().T.contiguous() + b.float()
    assert bool((z * 8 == torch.round(z * 8)).all()) and float(z.abs().max()) < 2 ** 20      # sums as exact as they are said to be
    want = ops.pack8(z)
    assert torch.equal(pre.scales, want.scales)
    assert torch.equal(pre.values.view(torch.uint8) & 0x7f, want.values.view(torch.uint8) & 0x7f)
    assert torch.equal(pre.values.float(), want.values.float())
    assert torch.equal(y, z.clamp_min(0).to(dtype))

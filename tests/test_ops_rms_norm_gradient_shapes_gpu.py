"""dip_rms_norm_grad over more rows than one launch takes both gradients of, in every
layout of a row: 4 to 64 lanes with a vector each or two, and a workgroup with one vector a
thread or two, each type, with and without gamma, dgamma, dx and what comes along.

Bounds, u = 2^-24, rstd as given: xh = t rstd and h = dy gamma are off by u of themselves, a
product by u more, and a row's sum has at most 16 terms of a thread, six steps in a wave, four
over the waves and a division: 32 u of the mean of |h xh|.  dx adds two roundings of the
product xh dot, one of the difference, one of the product with rstd and one of the sum with
dtotal.  dgamma's terms are off by 3 u; of up to 3000 rows a thread adds at most 12, a
workgroup joins 64, and at most 2048 of them are added by 16 lanes in 128 steps and joined in
16: 220 additions."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

if torch.cuda.is_available():
    from paper_2504_14145_amd import ops

F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
TYPES = [F32, BF16, F16]
u = 2.0 ** -24


@pytest.fixture(autouse=True)
def need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


def close(got, want, bound, dtype, what):
    half = torch.finfo(dtype).eps / 2
    tiny = 2.0 ** -25 if dtype is F16 else 2.0 ** -126
    limit = bound + half * (want.abs() + bound) + tiny
    off = (got.double() - want).abs()
    assert bool((off <= limit).all()), f"{what}: {float((off / limit).max())} of the bound"


def check(m, c, dtype, gamma, along, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    normal = lambda *s: torch.randn(s, generator=g, device="cuda")  # noqa: E731
    x, dy = (normal(m, c) * (1 + 5 * torch.rand(c, generator=g, device="cuda") ** 4)).to(dtype), normal(m, c).to(dtype)
    w = (1 + 0.3 * normal(c)).to(dtype) if gamma else None
    dt = normal(m, c).to(dtype) if along else None
    _, total, rstd, _ = ops.rms_norm(x, w)
    out = torch.full((m + 1, c + 3), 7.0, dtype=dtype, device="cuda")
    what = f"{m} x {c} {dtype} gamma {gamma} along {along}"
    dx, dg = ops.rms_norm_backward(dy, total, rstd, w, dtotal=dt, dx=out[:m, :c])
    r = rstd.double()[:, None]
    xh, d = total.double() * r, dy.double()
    h = d * w.double() if gamma else d
    dot, size = (h * xh).mean(1, keepdim=True), (h * xh).abs().mean(1, keepdim=True)
    want = r * (h - xh * dot)
    bound = r * (34 * u * xh.abs() * size + 5 * u * (h.abs() + (xh * dot).abs()))
    if along:
        want = want + dt.double()
        bound = bound + 2 * u * (want.abs() + dt.double().abs())
    close(dx, want, bound, dtype, what + " dx")
    assert bool((out[m] == 7.0).all()) and bool((out[:, c:] == 7.0).all())
    if not gamma:
        assert dg is None
        return
    wg, wb = (d * xh).sum(0), 223 * u * (d * xh).abs().sum(0)
    close(dg, wg, wb, dtype, what + " dgamma")
    acc = torch.full((c,), 0.5, device="cuda")
    none, got = ops.rms_norm_backward(dy, total, rstd, w, dtotal=dt, need_dx=False, dgamma=acc, accumulate=True)
    assert none is None and got is acc
    close(acc, wg + 0.5, wb + u, F32, what + " dgamma added to")
    # apart, together and in dtotal's place: the same bits
    assert torch.equal(ops.rms_norm_backward(dy, total, rstd, w, dtotal=dt, need_dgamma=False)[0], dx)
    if along:
        in_place, again = ops.rms_norm_backward(dy, total, rstd, w, dtotal=dt, dx=dt)
        assert in_place is dt and torch.equal(dt, dx) and torch.equal(again, dg)


# lanes a row 4, 8, 16, 32 and 64, these with two vectors (float32: a workgroup), a workgroup
# with one vector a thread and with two; whole vectors and rows that end inside one
COLS = (9, 32, 40, 64, 100, 128, 250, 256, 510, 512, 513, 700, 1024, 1027, 2051, 4096, 8192, 8200, 8203, 12345, 16384)


@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("c", COLS)
def test_many_rows(c, dtype):
    for i, (gamma, along) in enumerate(((True, True), (True, False), (False, True), (False, False))):
        m = (3000 if c < 3000 else 1000) - 37 * i
        check(m, c, dtype, gamma, along, c + i)


@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("c", (100, 700, 8200, 16384))
def test_where_one_launch_ends(c, dtype):
    """The most rows that one launch takes both gradients of, and one more."""
    most = 384 if dtype is F32 else 768
    for m in (most, most + 1):
        check(m, c, dtype, True, True, m)

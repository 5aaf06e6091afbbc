"""dip_rotary to the last bit: sines and cosines are those of 64 bits rounded once.

A pair (a, b) goes to (a c - b s, a s + b c), c and s within half a step of float32, 2^-24
of themselves, of their values: a 2^-24 |a c| + |b s| each.  The product b s is rounded, the
other product and the difference in one step or two: at most three roundings of 2^-24 of at
most |a c| + |b s| (1 + 2^-23) more.  So an output is within 4.01 2^-24 (|a c| + |b s|), and
half a step of its type, of its value."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

if torch.cuda.is_available():
    from paper_2504_14145_amd import ops

F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16


@pytest.fixture(autouse=True)
def need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


def turned(x, pos, freq, interleaved, inverse):
    """(value, sum of the magnitudes) in float64."""
    v = x.double()
    pairs = len(freq)
    a, b = (v[..., 0::2], v[..., 1::2]) if interleaved else v.chunk(2, -1)
    angle = (pos.double()[:, None] * freq)[:, None]
    c, s = angle.cos(), angle.sin() * (-1 if inverse else 1)
    join = (lambda p, q: torch.stack((p, q), -1).flatten(-2)) if interleaved else (lambda p, q: torch.cat((p, q), -1))
    return join(a * c - b * s, a * s + b * c), join((a * c).abs() + (b * s).abs(), (a * s).abs() + (b * c).abs()), pairs


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("pos_type", [torch.int32, torch.int64, F32])
def test_angles_of_64_bits(pos_type, interleaved):
    """Small and far positions, of either sign."""
    g = torch.Generator(device="cuda").manual_seed(3)
    q = torch.randn((3000, 3, 128), generator=g, device="cuda")
    freq, axis = ops.rotary_frequencies((64,))
    top = 20 if pos_type is F32 else 24
    pos = torch.randint(-1 << top, 1 << top, (3000,), generator=g, device="cuda")
    pos[:1000] %= 512
    pos = pos.to(pos_type) * (0.375 if pos_type is F32 else 1)
    for call, inverse in ((ops.rotary, False), (ops.rotary_backward, True)):
        got = call(q, pos, freq, axis, interleaved=interleaved).double()
        want, size, _ = turned(q, pos, freq, interleaved, inverse)
        # the angle's own roundings in float64: 2^-52 of it, times a turn's radians
        far = 2.0 ** -51 * float((pos.double().abs().max() * freq.max()))
        assert bool(((got - want).abs() <= (4.01 * 2.0 ** -24 + 0) * size + far * 8).all())


def test_sine_and_cosine_alone():
    """Pairs (1, 0): the outputs are the cosine and the sine themselves, within half a
    step, over the whole turn and beside the angles at which either is 0."""
    n = 1 << 16
    q = torch.zeros((n, 1, 2), device="cuda")
    q[..., 0] = 1
    axis = torch.zeros(1, dtype=torch.int32, device="cuda")
    quarter = torch.pi / 2
    for base, step in ((0.0, 1e-4), (-4.0, 1.3e-4), (0.0, 1e-9), (quarter, 1e-9), (-quarter, 1e-8), (2 * quarter, 1e-8),
                       (quarter / 2, 1e-8), (1e5, 1e-3)):
        freq = torch.tensor([step], dtype=torch.float64, device="cuda")
        pos = (torch.arange(n, device="cuda") - n // 2 + round(base / step)).long()
        angle = pos.double() * freq
        got = ops.rotary(q, pos, freq, axis)[:, 0].double()
        far = 2.0 ** -51 * (abs(base) + step * n)              # of the angle in float64, on either side
        for i, want in enumerate((angle.cos(), angle.sin())):
            # half a step, a 2^-8th of it for what is summed before the rounding
            bound = 2.0 ** -24 * (1 + 2.0 ** -8) * want.abs() + far
            assert bool(((got[:, i] - want).abs() <= bound).all()), (base, step, i)


@pytest.mark.parametrize("dtype", [BF16, F16], ids=str)
def test_outputs_of_16_bits_are_rounded_once(dtype):
    g = torch.Generator(device="cuda").manual_seed(4)
    q = torch.randn((2000, 4, 80), generator=g, device="cuda").to(dtype)
    freq, axis = ops.rotary_frequencies((40,))
    pos = torch.randint(0, 1 << 20, (2000,), generator=g, device="cuda")
    got = ops.rotary(q, pos, freq, axis).double()
    want, size, _ = turned(q, pos, freq, False, False)
    tiny = 2.0 ** -25 if dtype is F16 else 0.0
    assert bool(((got - want).abs() <= torch.finfo(dtype).eps / 2 * want.abs() + 4.01 * 2.0 ** -24 * size * (1 + 2.0 ** -8)
                 + 2.0 ** -30 + tiny).all())

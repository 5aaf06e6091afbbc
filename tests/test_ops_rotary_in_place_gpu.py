"""Rotary positions in their input's place where heads end inside a vector: what two threads
of different waves both turn comes out once turned."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

if torch.cuda.is_available():
    from paper_2504_14145_amd import ops

BF16, F16, F32 = torch.bfloat16, torch.float16, torch.float32


@pytest.fixture(autouse=True)
def need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


# pairs that are no multiple of a vector, a workgroup a token or several tokens, heads in
# shares of a token, and whole vectors
@pytest.mark.parametrize("t,heads,keys,dim", [(4000, 28, 28, 36), (3000, 40, 8, 42), (9000, 3, 2, 20), (500, 120, 40, 26),
                                              (700, 200, 0, 130), (2000, 28, 28, 128), (6000, 1, 1, 14), (300, 5, 4, 2046)])
@pytest.mark.parametrize("dtype", [BF16, F16, F32], ids=str)
@pytest.mark.parametrize("interleaved", [False, True])
def test_in_place_has_the_bits_of_apart(t, heads, keys, dim, dtype, interleaved):
    g = torch.Generator(device="cuda").manual_seed(dim)
    qk = torch.randn((t, heads + keys, dim), generator=g, device="cuda").to(dtype)
    pos = torch.randint(0, 100000, (t, 2), generator=g, device="cuda")
    pairs = dim // 2
    freq, axis = ops.rotary_frequencies((pairs // 2, pairs - pairs // 2))
    q, k = qk[:, :heads], qk[:, heads:] if keys else None
    for call, name in ((ops.rotary, "k"), (ops.rotary_backward, "dk")):
        want = call(q, pos, freq, axis, **{name: k}, interleaved=interleaved)
        got = call(q, pos, freq, axis, **{name: k}, interleaved=interleaved, out=q, out_k=k)
        assert torch.equal(want[0] if keys else want, q) and (not keys or torch.equal(want[1], k))
        assert (got[0] if keys else got) is q

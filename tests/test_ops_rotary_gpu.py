"""dip_rotary against its plain 64-bit form."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from kept_reference import rotary  # noqa: E402
from ops_reference import assert_close  # noqa: E402

if torch.cuda.is_available():
    from paper_2504_14145_amd import ops

F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
TYPES = [F32, BF16, F16]


@pytest.fixture(autouse=True)
def need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


def inputs(t, heads, keys, dim, dtype, seed):
    g = torch.Generator().manual_seed(seed)
    q = torch.randn((t, heads, dim), generator=g).to(dtype)
    k = torch.randn((t, keys, dim), generator=g).to(dtype) if keys else None
    return g, q, k


def check(t, heads, keys, dim, sections, dtype, interleaved=False, shared=False, pos_type=torch.int32, most=2000, seed=1):
    g, q, k = inputs(t, heads, keys, dim, dtype, seed)
    pos = torch.randint(0, most, (t, len(sections)), generator=g).to(pos_type)
    if pos_type is F32:
        pos = pos * 0.375 - 40
    freq, axis = ops.rotary_frequencies(sections, shared=shared)
    for call, inverse in ((ops.rotary, False), (ops.rotary_backward, True)):
        args = dict(interleaved=interleaved)
        if keys:
            args["dk" if inverse else "k"] = k.cuda()
        got = call(q.cuda(), pos.cuda(), freq, axis, **args)
        for name, x, y in (("q", q, got[0] if keys else got),) + ((("k", k, got[1]),) if keys else ()):
            want, bound = rotary(x, pos, freq, axis, interleaved, inverse)
            assert_close(y, want, bound, dtype, f"{name} {t} x {heads} + {keys} x {dim} {sections} {dtype} inverse {inverse}")
            rest = 2 * sum(sections)
            assert torch.equal(y[..., rest:].cpu(), x[..., rest:])


@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("dim,sections", [(128, (16, 24, 24)), (112, (28, 28)), (64, (32,)), (72, (12, 12, 12)), (20, (5, 5)),
                                          (6, (1, 1, 1)), (2, (1,)), (256, (32, 32, 32, 32)), (42, (10, 11)), (2048, (512, 512))])
def test_dims(dim, sections, interleaved, dtype):
    check(13, 5, 2, dim, sections, dtype, interleaved, seed=dim)


@pytest.mark.parametrize("t,heads,keys", [(1, 1, 0), (1, 32, 8), (1, 64, 64), (2, 3, 1), (149, 32, 8), (1025, 16, 16), (4100, 2, 2),
                                          (3, 130, 7), (700, 28, 28)])
@pytest.mark.parametrize("interleaved", [False, True])
def test_tokens_and_heads(t, heads, keys, interleaved):
    check(t, heads, keys, 64, (8, 12, 12), BF16, interleaved, seed=t)


@pytest.mark.parametrize("pos_type", [torch.int32, torch.int64, F32])
@pytest.mark.parametrize("shared", [False, True])
def test_positions(pos_type, shared):
    check(70, 3, 1, 48, (8, 8, 8), F32, shared=shared, pos_type=pos_type)


def test_far_positions_keep_their_angles():
    """Beyond 2^24, where float32 has no odd numbers, and far negative ones."""
    _, q, _ = inputs(4, 2, 0, 32, F32, 3)
    freq, axis = ops.rotary_frequencies((16,))
    pos = torch.tensor([[2 ** 24 + 1], [10 ** 9 + 7], [-(10 ** 8) - 3], [2 ** 31 - 1]])
    for t in (torch.int64, torch.int32):
        got = ops.rotary(q.cuda(), pos.to(t).cuda(), freq, axis)
        assert_close(got, *rotary(q, pos, freq, axis, False), F32, str(t))


@pytest.mark.parametrize("dim", [40, 33])
@pytest.mark.parametrize("interleaved", [False, True])
def test_heads_that_turn_in_part(dim, interleaved):
    check(50, 4, 2, dim, (4, 6), BF16, interleaved)
    check(50, 4, 0, dim, (3,), F16, interleaved)
    check(5, 4, 1, dim, (), F32, interleaved)


def test_axes_that_positions_do_not_have():
    _, q, _ = inputs(9, 2, 0, 16, F32, 5)
    freq = torch.ones(8, dtype=torch.float64, device="cuda")
    axis = torch.tensor([0, 1, -1, 2, 1, 5, 0, -7], dtype=torch.int32, device="cuda")
    pos = torch.arange(18).reshape(9, 2).to(torch.int32)
    got = ops.rotary(q.cuda(), pos.cuda(), freq, axis)
    assert_close(got, *rotary(q, pos, freq, axis, False), F32, "axes")
    still = [j + s for j in (2, 3, 5, 7) for s in (0, 8)]
    assert torch.equal(got[..., still].cpu(), q[..., still])


@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("interleaved", [False, True])
def test_views_of_one_array_and_in_place(dtype, interleaved):
    """q and k as slices of one product's output, heads outside tokens, odd strides, and
    outputs that are the inputs: the same bits."""
    t, h, k, d = 61, 6, 2, 24
    g = torch.Generator().manual_seed(9)
    qkv = torch.randn((t, h + 2 * k, d + 1), generator=g).to(dtype).cuda()
    pos = torch.randint(0, 500, (t, 2), generator=g).cuda()
    freq, axis = ops.rotary_frequencies((5, 6))
    q, kk = qkv[:, :h, :d], qkv[:, h:h + k, :d]
    want = ops.rotary(q.contiguous(), pos, freq, axis, k=kk.contiguous(), interleaved=interleaved)
    got = ops.rotary(q, pos, freq, axis, k=kk, interleaved=interleaved)
    assert all(torch.equal(a, b) for a, b in zip(want, got))
    outside = q.transpose(0, 1).contiguous().transpose(0, 1)
    out = torch.empty((h, t, d), dtype=dtype, device="cuda").transpose(0, 1)
    assert torch.equal(ops.rotary(outside, pos, freq, axis, interleaved=interleaved, out=out), want[0])
    across = pos.T.contiguous().T           # [axes][tokens] in memory
    assert torch.equal(ops.rotary(q, across, freq, axis, interleaved=interleaved), want[0])
    keep = qkv.clone()
    a, b = ops.rotary(q, pos, freq, axis, k=kk, interleaved=interleaved, out=q, out_k=kk)
    assert a is q and b is kk and torch.equal(q, want[0]) and torch.equal(kk, want[1])
    assert torch.equal(qkv[:, h + k:], keep[:, h + k:]) and torch.equal(qkv[..., d:], keep[..., d:])


def test_gradient_is_the_transposed_turn():
    """<rotary(q), dy> = <q, rotary_backward(dy)>, and turning back gives q."""
    _, q, dy = inputs(40, 3, 3, 64, F32, 11)
    freq, axis = ops.rotary_frequencies((16, 16))
    pos = torch.randint(0, 5000, (40, 2), generator=torch.Generator().manual_seed(2)).cuda()
    y, dq = ops.rotary(q.cuda(), pos, freq, axis), ops.rotary_backward(dy.cuda(), pos, freq, axis)
    a, b = (y.double() * dy.cuda().double()).sum(), (q.cuda().double() * dq.double()).sum()
    assert abs(float(a - b)) <= 2.0 ** -19 * float((q.abs().double() * dy.abs().double()).sum()) * 2
    back = ops.rotary_backward(y, pos, freq, axis).cpu()
    pair = torch.hypot(*q.chunk(2, -1))
    assert bool(((back - q).abs() <= 2.0 ** -18 * torch.cat((pair, pair), -1)).all())


def test_one_axis_without_a_dimension_and_one_position_for_all():
    _, q, _ = inputs(10, 2, 0, 16, BF16, 12)
    freq, axis = ops.rotary_frequencies((8,))
    pos = torch.arange(10)
    assert torch.equal(ops.rotary(q.cuda(), pos.cuda(), freq, axis), ops.rotary(q.cuda(), pos[:, None].cuda(), freq, axis))
    one = torch.tensor([[7]]).cuda().expand(10, 1)
    want = ops.rotary(q.cuda(), torch.full((10, 1), 7).cuda(), freq, axis)
    assert torch.equal(ops.rotary(q.cuda(), one, freq, axis), want)


def test_empty_and_refusals():
    q = torch.zeros((5, 2, 16), device="cuda")
    freq, axis = ops.rotary_frequencies((8,))
    pos = torch.zeros((5, 1), dtype=torch.int32, device="cuda")
    assert ops.rotary(q[:0], pos[:0], freq, axis).shape == (0, 2, 16)
    assert ops.rotary(q[:, :0], pos, freq, axis, k=q)[1].shape == (5, 2, 16)
    for call in (lambda: ops.rotary(q[0], pos, freq, axis), lambda: ops.rotary(q, pos[:4], freq, axis),
                 lambda: ops.rotary(q, pos.double(), freq, axis), lambda: ops.rotary(q, pos.cpu(), freq, axis),
                 lambda: ops.rotary(q, pos, freq.float(), axis), lambda: ops.rotary(q, pos, freq, axis.long()),
                 lambda: ops.rotary(q, pos, freq, axis[:7]), lambda: ops.rotary(q[..., :14], pos, freq, axis),
                 lambda: ops.rotary(q, pos, freq, axis, k=q[:4]), lambda: ops.rotary(q, pos, freq, axis, k=q.half()),
                 lambda: ops.rotary(q, pos, freq, axis, out_k=q), lambda: ops.rotary(q, pos, freq, axis, out=q[:4]),
                 lambda: ops.rotary(q.transpose(1, 2), pos, freq, axis)):
        with pytest.raises(ValueError):
            call()
    with pytest.warns(UserWarning, match="rotary records no gradients"):
        ops.rotary(q.clone().requires_grad_(True), pos, freq, axis)


def test_graph_and_stream():
    t = 500
    q, k = torch.randn((t, 8, 128), device="cuda").to(BF16), torch.randn((t, 2, 128), device="cuda").to(BF16)
    pos = torch.randint(0, 900, (t, 3), device="cuda")
    freq, axis = ops.rotary_frequencies((16, 24, 24))
    oq, ok = torch.empty_like(q), torch.empty_like(k)
    graph = torch.cuda.CUDAGraph()
    ops.rotary(q, pos, freq, axis, k=k, out=oq, out_k=ok)
    with torch.cuda.graph(graph):
        ops.rotary(q, pos, freq, axis, k=k, out=oq, out_k=ok)
    for _ in range(3):
        q.normal_()
        pos.random_(0, 4000)
        graph.replay()
        torch.cuda.synchronize()
        a, b = ops.rotary(q, pos, freq, axis, k=k)
        assert torch.equal(a, oq) and torch.equal(b, ok)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    a, b = ops.rotary(q, pos, freq, axis, k=k, stream=side)
    c, d = ops.rotary_backward(a, pos, freq, axis, dk=b, stream=side.cuda_stream)
    side.synchronize()
    assert torch.equal(a, oq) and torch.equal(b, ok)
    assert torch.equal(c, ops.rotary_backward(oq, pos, freq, axis)) and d.shape == k.shape

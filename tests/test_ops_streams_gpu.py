"""Calls on a stream other than torch's current one: whose memory they work in."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

if torch.cuda.is_available():
    from paper_2504_14145_amd import ops

BF16 = torch.bfloat16


@pytest.fixture(autouse=True)
def need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


def owner(t):
    """Handle of the stream from whose pool the allocator took t."""
    for s in torch.cuda.memory_snapshot():
        if s["address"] <= t.data_ptr() < s["address"] + s["total_size"]:
            return s["stream"]
    raise AssertionError("not the allocator's")


def calls(side):
    """Every operator where it needs a workspace and allocates its results."""
    x, dy = torch.randn((300, 515), device="cuda").to(BF16), torch.randn((300, 72), device="cuda").to(BF16)
    w, pre = torch.randn((72, 515), device="cuda").to(BF16), torch.randn((300, 72), device="cuda").to(BF16)
    v = torch.randn((2, 5000, 64), device="cuda")
    gamma = torch.ones(64, device="cuda")
    drop = ops.Dropout(0.1, 3)
    _, mean, rstd = ops.group_norm(v, 8, gamma, gamma)
    torch.cuda.synchronize()
    return (lambda: ops.linear(x, w, act="gelu", dropout=drop, stream=side),
            lambda: ops.linear_backward(dy, x, w, act="gelu", dropout=drop, pre=pre, stream=side),
            lambda: ops.dropout_add(dy, drop, stream=side),
            lambda: ops.group_norm(v, 8, gamma, gamma, stream=side),
            lambda: ops.group_norm_backward(v, v, mean, rstd, 8, gamma, gamma, stream=side))


@pytest.mark.parametrize("raw", [False, True])
def test_results_and_workspaces_are_of_the_stream_that_uses_them(monkeypatch, raw):
    """With no wait between the streams: everything given is ready, and nothing else
    may come from the current stream, whose pending work could still use it."""
    spaces = []
    take = torch.empty
    side = torch.cuda.Stream()
    for n, call in enumerate(calls(side.cuda_stream if raw else side)):
        want = calls(None)[n]()     # loads the library, too
        monkeypatch.setattr(ops, "_empty", lambda *a, **k: spaces.append(take(*a, **k)) or spaces[-1])
        spaces.clear()
        got = call()
        monkeypatch.undo()
        side.synchronize()
        assert bool(spaces) == (n != 2), n
        for t in (*spaces, *(got if isinstance(got, tuple) else (got,))):
            assert owner(t) == side.cuda_stream, n
        del want


def test_results_on_a_stream_whose_pool_is_fresh_beside_pending_work():
    """The current stream still works in blocks that it has freed; calls on another
    one, that wait for nothing, give the same bits."""
    side = torch.cuda.Stream()
    x, w = torch.randn((4096, 515), device="cuda").to(BF16), torch.randn((512, 515), device="cuda").to(BF16)
    pre, dy = torch.randn((4096, 512), device="cuda").to(BF16), torch.randn((4096, 512), device="cuda").to(BF16)
    want = ops.linear_backward(dy, x, w, act="gelu", pre=pre)
    torch.cuda.synchronize()
    for _ in range(3):
        for _ in range(40):
            for size in (1 << 20, 1 << 22, 1 << 24):
                torch.full((size,), -1.0, device="cuda")     # freed while it is written
        got = ops.linear_backward(dy, x, w, act="gelu", pre=pre, stream=side)
        side.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(want, got))
    torch.cuda.synchronize()

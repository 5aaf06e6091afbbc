"""Layer blocks that run the norm, the products, the rotary positions and the 8-bit
activations together: gradients against 64 bits, kept, kept in 8 bits and recomputed."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from kept_reference import RmsNorm  # noqa: E402
from ops_reference import mask  # noqa: E402

if torch.cuda.is_available():
    from paper_2504_14145_amd import ops
    from paper_2504_14145_amd.stage import Block, Projection

BF16, F16 = torch.bfloat16, torch.float16
# bf16 intermediates: about five roundings of at most 2^-8 on the way of a value, averaged
# by the sums they go through: 2^-6 of the result's norm (fp16 the less).  Kept in 8 bits a
# value is off by at most 2^-4 of it, evenly spread within that 2^-4 / sqrt(3) of a sum's norm.
NEAR = {True: 2.0 ** -6, False: 2.0 ** -6, 8: 2.0 ** -6 + 2.0 ** -4 / 3 ** 0.5}


@pytest.fixture(autouse=True)
def need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


def near(got, want, what, limit):
    got = got.cpu().double()
    assert float((got - want).norm()) <= limit * float(want.norm()), (what, float((got - want).norm() / want.norm()))


def norm64(x, gamma, beta):
    if beta is None:
        return x / torch.sqrt((x * x).mean(1, keepdim=True) + 1e-5) * gamma
    d = x - x.mean(1, keepdim=True)
    return d / torch.sqrt((d * d).mean(1, keepdim=True) + 1e-5) * gamma + beta


def plain_block(block, x, dy, seed, row0):
    par = {n: getattr(block, n).cpu().double().requires_grad_(True) for n in block.grads}
    xv = x.cpu().double().requires_grad_(True)
    z = norm64(xv, par["gamma"], par.get("beta")) @ par["w1"].T + par["b1"]
    u = z if block.act == "none" else z * torch.sigmoid(z if block.act == "silu" else
                                                        2 * 0.7978845608028654 * (z + 0.044715 * z ** 3))
    v = u @ par["w2"].T + par["b2"]
    if block.p:
        drop = ops.Dropout(block.p, seed, offset=block.layer, row0=row0)
        v = torch.where(mask(drop, x.shape[0], block.hidden), v * drop.scale, 0.0)
    y = xv + v
    y.backward(dy.cpu().double())
    return y.detach(), xv.grad, {n: p.grad for n, p in par.items()}


@pytest.mark.parametrize("keep", [True, 8, False])
@pytest.mark.parametrize("t,h,f,p,act,norm,dtype", [
    (1, 64, 96, 0.0, "silu", "rms", "bf16"), (37, 136, 264, 0.25, "gelu", "rms", "bf16"),
    (300, 256, 512, 0.1, "silu", "rms", "fp16"), (300, 256, 512, 0.1, "gelu", "layer", "bf16"),
    (130, 200, 328, 0.0, "none", "rms", "bf16")])
def test_block_gradients(t, h, f, p, act, norm, dtype, keep):
    dtype = BF16 if dtype == "bf16" else F16
    block = Block(h, f, act=act, p=p, layer=3, seed=t, norm=norm, dtype=dtype)
    g = torch.Generator().manual_seed(t)
    block.b1.copy_(torch.randn(f, generator=g) * 0.3)
    block.gamma.copy_(1 + 0.2 * torch.randn(h, generator=g))
    x, dy = (torch.randn((t, h), generator=g).to(dtype).cuda() for _ in range(2))
    assert ("beta" in block.grads) == (norm == "layer")
    y, saved = block.forward(x, seed=11, row0=5, keep=keep)
    dx = block.backward(dy, saved)
    wy, wdx, wg = plain_block(block, x, dy, 11, 5)
    near(y, wy, "y", 2.0 ** -6)
    near(dx, wdx, "dx", NEAR[keep])
    for n, v in block.grads.items():
        near(v, wg[n], n, NEAR[keep])


def held(saved, but):
    """Bytes of a forward's saved tensors, its input not counted."""
    total = 0
    for v in saved:
        if isinstance(v, tuple):
            total += held(v, but)
        elif isinstance(v, ops.Packed8):
            total += v.values.numel() + v.scales.numel()
        elif isinstance(v, torch.Tensor) and v is not but:
            total += v.numel() * v.element_size()
    return total


def test_what_a_block_keeps():
    t, h, f = 64, 256, 1024
    block = Block(h, f, norm="rms")
    x = torch.randn((t, h), device="cuda").to(BF16)
    bytes_of = {k: held(block.forward(x, keep=k)[1], x) for k in (True, 8, False)}
    assert bytes_of == {True: t * (2 * h + 4 * f) + 4 * t, 8: t * (h + f) * 33 // 32 + 4 * t, False: 0}
    for keep in (2, "8", None):
        with pytest.raises(ValueError):
            block.forward(x, keep=keep)
    with pytest.raises(ValueError):
        Block(h, f, norm="batch")


def test_the_8_bit_block_is_its_operators_in_turn():
    """Bit by bit what the calls on restored activations give."""
    t, h, f = 90, 128, 200
    block = Block(h, f, act="silu", norm="rms", seed=3)
    g = torch.Generator().manual_seed(3)
    x, dy = (torch.randn((t, h), generator=g).to(BF16).cuda() for _ in range(2))
    _, saved = block.forward(x, keep=8)
    n8, _, rstd, pre8, u = saved[3]
    assert u is None
    dx = block.backward(dy, saved)
    pre = ops.unpack8(pre8)
    du, dw2, _ = ops.linear_backward(dy, ops.unpack8(pre8, act="silu"), block.w2, dw=torch.zeros((h, f), device="cuda"),
                                     db=torch.zeros(h, device="cuda"))
    dn, dw1, db1 = ops.linear_backward(du, ops.unpack8(n8), block.w1, act="silu", pre=pre, dw=torch.zeros((f, h), device="cuda"),
                                       db=torch.zeros(f, device="cuda"))
    want, dgamma = ops.rms_norm_backward(dn, x, rstd, block.gamma, dtotal=dy)
    assert torch.equal(dx, want) and torch.equal(block.grads["gamma"].to(BF16), dgamma)
    for name, v in (("w1", dw1), ("w2", dw2), ("b1", db1)):
        assert torch.equal(block.grads[name], v), name


def turn64(x, pos, freq, axis, interleaved):
    pairs = freq.shape[0]
    j = torch.arange(pairs)
    first = 2 * j if interleaved else j
    second = first + (1 if interleaved else pairs)
    angle = pos.double()[:, axis.long()] * freq
    c, s = angle.cos()[:, None], angle.sin()[:, None]
    a, b = x[..., first], x[..., second]
    parts = torch.cat((a * c - b * s, a * s + b * c, x[..., 2 * pairs:]), -1)
    order = torch.cat((first, second, torch.arange(2 * pairs, x.shape[-1])))
    return parts[..., torch.argsort(order)]


@pytest.mark.parametrize("keep", [True, 8, False])
@pytest.mark.parametrize("t,h,heads,keys,dim,sections,inter", [
    (1, 64, 2, 1, 32, (4, 6, 6), False), (70, 136, 4, 2, 40, (10, 10), True), (300, 256, 4, 4, 64, (8, 8, 8), False)])
def test_projection_gradients(t, h, heads, keys, dim, sections, inter, keep):
    block = Projection(h, heads, keys, dim, sections, interleaved=inter, seed=t)
    g = torch.Generator().manual_seed(t)
    block.b.copy_(torch.randn(block.b.shape, generator=g) * 0.3)
    block.gamma.copy_(1 + 0.2 * torch.randn(h, generator=g))
    x, r, dt = (torch.randn((t, h), generator=g).to(BF16).cuda() for _ in range(3))
    pos = torch.randint(0, 200, (t, len(sections)), generator=g).cuda()
    q, k, v, total, saved = block.forward(x, pos, residual=r, keep=keep)
    dq, dk, dv = (torch.randn(s.shape, generator=g).to(BF16).cuda() for s in (q, k, v))
    dx = block.backward(dq, dk, dv, saved, dtotal=dt)
    # 64 bits, from the rounded stream of residuals
    par = {n: getattr(block, n).cpu().double().requires_grad_(True) for n in block.grads}
    assert torch.equal(total.cpu(), RmsNorm(x, r, None, 1e-5).total)
    tv = total.cpu().double().requires_grad_(True)
    z = (norm64(tv, par["gamma"], None) @ par["w"].T + par["b"]).view(t, -1, dim)
    freq, axis = block.frequencies.cpu(), block.axis.cpu()
    wq, wk, wv = (turn64(z[:, :heads], pos.cpu(), freq, axis, inter),
                  turn64(z[:, heads:heads + keys], pos.cpu(), freq, axis, inter), z[:, heads + keys:])
    loss = sum((a * b.cpu().double()).sum() for a, b in ((wq, dq), (wk, dk), (wv, dv), (tv, dt)))
    loss.backward()
    for name, a, b in (("q", q, wq), ("k", k, wk), ("v", v, wv)):
        near(a, b.detach(), name, 2.0 ** -6)
    near(dx, tv.grad, "dx", 2.0 ** -6)
    for n, p in par.items():
        near(block.grads[n], p.grad, n, NEAR[keep])


@pytest.mark.parametrize("keep", [True, 8, False])
def test_a_piece_without_tokens(keep):
    block, pro = Block(64, 128, act="silu", norm="rms"), Projection(64, 2, 1, 16, (4, 4))
    x, pos = torch.empty((0, 64), dtype=BF16, device="cuda"), torch.empty((0, 2), dtype=torch.int32, device="cuda")
    y, saved = block.forward(x, keep=keep)
    assert y.shape == (0, 64) and block.backward(y, saved).shape == (0, 64)
    q, k, v, total, saved = pro.forward(x, pos, residual=x, keep=keep)
    assert q.shape == (0, 2, 16) and k.shape == v.shape == (0, 1, 16)
    assert pro.backward(q, k, v, saved, dtotal=x).shape == (0, 64)
    for g in (*block.grads.values(), *pro.grads.values()):
        assert not g.any()


def test_shares_of_a_projection_add_up():
    h, heads, keys, dim, t = 96, 4, 2, 24, 50
    whole = Projection(h, heads, keys, dim, (4, 8), seed=1)
    g = torch.Generator().manual_seed(2)
    whole.gamma.copy_(1 + 0.2 * torch.randn(h, generator=g))
    x, r, dt = (torch.randn((t, h), generator=g).to(BF16).cuda() for _ in range(3))
    pos = torch.randint(0, 200, (t, 2), generator=g).cuda()
    q, k, v, _, saved = whole.forward(x, pos, residual=r)
    d = [torch.randn(s.shape, generator=g).to(BF16).cuda() for s in (q, k, v)]
    dx = whole.backward(*d, saved, dtotal=dt)
    parts, dx_sum, gamma = [], 0, 0
    rows = whole.w.view(-1, dim, h)
    for rank in range(2):
        share = Projection(h, heads, keys, dim, (4, 8), tp=2, rank=rank)
        mine = (slice(rank * 2, rank * 2 + 2), slice(4 + rank, 5 + rank), slice(6 + rank, 7 + rank))
        share.w.copy_(torch.cat([rows[m] for m in mine]).view(-1, h))
        share.gamma.copy_(whole.gamma)
        sq, sk, sv, _, saved = share.forward(x, pos, residual=r)
        parts.append((sq, sk, sv))
        sd = share.backward(d[0][:, rank * 2:rank * 2 + 2], d[1][:, rank:rank + 1], d[2][:, rank:rank + 1], saved, dtotal=dt)
        dx_sum, gamma = dx_sum + sd.float(), gamma + share.grads["gamma"]
    for i, want in enumerate((q, k, v)):
        assert torch.equal(torch.cat([p[i] for p in parts], 1), want)
    near(dx_sum, dx.cpu().double(), "dx", 2.0 ** -6)
    near(gamma, whole.grads["gamma"].cpu().double(), "gamma", 2.0 ** -6)
    for bad in (dict(tp=3), dict(tp=2, rank=2)):
        with pytest.raises(ValueError):
            Projection(h, heads, keys, dim, (4, 8), **bad)
    with pytest.raises(ValueError):
        Projection(h, heads, keys, dim, (8, 8))


def test_recomputed_projection_has_the_kept_ones_gradients():
    block = Projection(128, 4, 2, 32, (8, 8), seed=5)
    g = torch.Generator().manual_seed(5)
    x, r = (torch.randn((60, 128), generator=g).to(BF16).cuda() for _ in range(2))
    pos = torch.randint(0, 99, (60, 2), generator=g).cuda()
    got = []
    for keep in (True, False):
        for v in block.grads.values():
            v.zero_()
        q, k, v, total, saved = block.forward(x, pos, residual=r, keep=keep)
        got.append([q, k, v, total, block.backward(q, k, v, saved)] + [p.clone() for p in block.grads.values()])
    assert all(torch.equal(a, b) for a, b in zip(*got))


@pytest.mark.parametrize("keep", [True, 8])
def test_a_layers_pass_in_a_graph(keep):
    """Projection, then block, forward and backward, captured and replayed on other
    inputs beside eager passes."""
    pro, block = Projection(128, 4, 2, 32, (8, 8), seed=1), Block(128, 256, act="silu", p=0.1, norm="rms", seed=2)
    x, r = torch.randn((90, 128), device="cuda").to(BF16), torch.randn((90, 128), device="cuda").to(BF16)
    pos = torch.randint(0, 50, (90, 2), device="cuda")
    grads = list(pro.grads.values()) + list(block.grads.values())

    def step():
        for v in grads:
            v.zero_()
        q, k, v, total, a = pro.forward(x, pos, residual=r, keep=keep)
        y, b = block.forward(total, seed=3, keep=keep)
        dt = block.backward(y, b)
        dx = pro.backward(q, k, v, a, dtotal=dt)
        return [y, dx] + [v.clone() for v in grads]

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step()
    for _ in range(3):
        x.normal_()
        pos.random_(0, 3000)
        graph.replay()
        torch.cuda.synchronize()
        got = [v.clone() for v in out]
        for a, b in zip(step(), got):
            assert torch.equal(a, b)
        torch.cuda.synchronize()

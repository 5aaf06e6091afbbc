"""A layer block of the stage operators: its gradients, recomputation, pieces of
a sample, and the way from times to a simulated schedule."""
import dataclasses

import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

import oracle  # noqa: E402
import workloads as W  # noqa: E402
from oracle import costmodel  # noqa: E402
from ops_reference import mask  # noqa: E402
from workloads.operators import N_KINDS, operator_table  # noqa: E402

if torch.cuda.is_available():
    import paper_2504_14145_amd as dip
    from paper_2504_14145_amd import calibrate, ops
    from paper_2504_14145_amd.stage import Block

BF16 = torch.bfloat16


@pytest.fixture(autouse=True)
def need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


def plain(block, x, dy, seed, row0):
    """y and the gradients in 64 bits, by torch's own differentiation."""
    t = x.shape[0]
    par = {n: getattr(block, n).cpu().double().requires_grad_(True) for n in block.grads}
    xv = x.cpu().double().requires_grad_(True)
    d = xv - xv.mean(1, keepdim=True)
    n = d / torch.sqrt((d * d).mean(1, keepdim=True) + 1e-5) * par["gamma"] + par["beta"]
    z = n @ par["w1"].T + par["b1"]
    u = z * torch.sigmoid(2 * 0.7978845608028654 * (z + 0.044715 * z ** 3))
    v = u @ par["w2"].T + par["b2"]
    if block.p:
        drop = ops.Dropout(block.p, seed, offset=block.layer, row0=row0)
        v = torch.where(mask(drop, t, block.hidden), v * drop.scale, 0.0)
    y = xv + v
    y.backward(dy.cpu().double())
    return y.detach(), xv.grad, {n: p.grad for n, p in par.items()}


def make(t, h, f, p, seed):
    block = Block(h, f, p=p, layer=3, seed=seed)
    g = torch.Generator().manual_seed(seed)
    block.b1.copy_(torch.randn(block.ffn, generator=g) * 0.3)
    block.gamma.copy_(1 + 0.2 * torch.randn(h, generator=g))
    block.beta.copy_(0.1 * torch.randn(h, generator=g))
    return block, torch.randn((t, h), generator=g).to(BF16).cuda(), torch.randn((t, h), generator=g).to(BF16).cuda()


def near(got, want, what):
    """bf16 intermediates: about five roundings of at most 2^-8 on the way of a value,
    independent of each other and averaged by the sums they go through: 2^-6 of
    the result's norm."""
    got, want = got.cpu().double(), want
    assert float((got - want).norm()) <= 2.0 ** -6 * float(want.norm()), what


@pytest.mark.parametrize("t,h,f,p", [(1, 64, 96, 0.0), (37, 136, 264, 0.25), (300, 256, 512, 0.1)])
def test_block_gradients(t, h, f, p):
    block, x, dy = make(t, h, f, p, t)
    y, saved = block.forward(x, seed=11, row0=5)
    dx = block.backward(dy, saved)
    wy, wdx, wg = plain(block, x, dy, 11, 5)
    near(y, wy, "y")
    near(dx, wdx, "dx")
    for n, g in block.grads.items():
        near(g, wg[n], n)


def test_recomputed_gradients_are_the_kept_ones():
    block, x, dy = make(130, 256, 384, 0.3, 4)
    got = []
    for keep in (True, False):
        for g in block.grads.values():
            g.zero_()
        y, saved = block.forward(x, seed=9, keep=keep)
        assert keep or saved[3] is None
        got.append([y, block.backward(dy, saved)] + [g.clone() for g in block.grads.values()])
    assert all(torch.equal(a, b) for a, b in zip(*got))


def test_pieces_of_a_sample_add_up():
    block, x, dy = make(96, 128, 256, 0.4, 6)
    y, saved = block.forward(x, seed=2)
    dx = block.backward(dy, saved)
    whole = {n: g.clone() for n, g in block.grads.items()}
    for g in block.grads.values():
        g.zero_()
    for lo, hi in ((0, 40), (40, 41), (41, 96)):
        py, saved = block.forward(x[lo:hi], seed=2, row0=lo)
        pdx = block.backward(dy[lo:hi], saved)
        near(py, y[lo:hi].cpu().double(), "y")
        near(pdx, dx[lo:hi].cpu().double(), "dx")
    for n, g in block.grads.items():
        near(g, whole[n].cpu().double(), n)


def test_measured_costs_run_a_schedule():
    """measure, fit, the cost tables against their oracle, and the simulator on
    them against its own."""
    prob = W.make_problem(2)
    samples = calibrate.measure([(512, 2048)], [33, 512], tp=1, repeats=3)
    assert len(samples) == 12 and all(s.seconds > 0 for s in samples)
    base = np.tile([1e-15, 1e-13, 1e-11], (N_KINDS, 1))
    coef = calibrate.fit(samples, base)
    assert np.isfinite(coef).all() and (coef > 0).all()
    assert calibrate.accuracy(samples, coef) >= calibrate.accuracy(samples, base)
    rows = operator_table(prob)
    table = dip.DeviceOpTable(rows, N_KINDS)
    out = torch.empty((1, table.n_items), dtype=torch.int32, device="cuda")
    dip.cost_tables(table, torch.from_numpy(coef[None].copy()).cuda(), out)
    costs = out[0].cpu().numpy()
    np.testing.assert_array_equal(costs, costmodel.cost_tables(rows, coef[None])[0])
    prob = dataclasses.replace(prob, op_cost=costs[:prob.n_total], edge_comm=costs[prob.n_total:])
    orders = W.generator_for(prob, 2).generate(0, 200)
    sim = dip.Sim(prob)
    ms, bub, pk, fl = sim.evaluate(torch.from_numpy(np.ascontiguousarray(orders)).cuda())
    want = oracle.evaluate(prob, orders, threads=4)
    np.testing.assert_array_equal(ms.cpu().numpy(), want.makespan)
    np.testing.assert_array_equal(fl.cpu().numpy(), want.flags)

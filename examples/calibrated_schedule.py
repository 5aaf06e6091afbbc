"""Plans a pipeline with costs measured on this card.

    python examples/calibrated_schedule.py [--workload 2] [--candidates 4096]

1. runs one layer block of each module's sizes (the MLP without a gate) forward
   and backward with the stage operators, kept and recomputed, and checks that both
   give the same gradients;
2. times the operators at the workload's token counts and fits the cost tables'
   coefficients to them (kinds without an operator here keep a factor of 1 on
   the card's nominal rates);
3. builds the cost table of every pipeline stage and edge with them, simulates a
   batch of candidate schedules on those costs and reports the best.
"""
import argparse
import dataclasses
import os
import sys

import numpy as np
import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import paper_2504_14145_amd as dip  # noqa: E402
import workloads as W  # noqa: E402
from paper_2504_14145_amd import calibrate  # noqa: E402
from paper_2504_14145_amd.stage import Block  # noqa: E402
from workloads.operators import N_KINDS, SEGMENT_MODELS, operator_table  # noqa: E402

MI355X = {"flops": 2.5e15, "mem_bw": 8e12, "net_bw": 153e9}


def run_block(spec, tokens, tp):
    block = Block(spec.hidden, spec.ffn, p=0.1, tp=tp)
    x = torch.randn((tokens, spec.hidden), device="cuda").bfloat16()
    dy = torch.randn_like(x)
    grads = []
    for keep in (True, False):
        for g in block.grads.values():
            g.zero_()
        _, saved = block.forward(x, seed=7, keep=keep)
        dx = block.backward(dy, saved)
        grads.append([dx] + [g.clone() for g in block.grads.values()])
    same = all(torch.equal(a, b) for a, b in zip(*grads))
    print(f"{spec.name}: {tokens} tokens, recomputed gradients {'equal' if same else 'DIFFER FROM'} the kept ones")
    return same


def main():
    ap = argparse.ArgumentParser()
    ap.add_argument("--workload", type=int, default=2)
    ap.add_argument("--candidates", type=int, default=4096)
    ap.add_argument("--tp", type=int, default=4)
    a = ap.parse_args()
    prob = W.make_problem(a.workload)
    names = [s.name for s in W.CONFIGS[a.workload].segments]
    specs = {SEGMENT_MODELS[n].name: SEGMENT_MODELS[n] for n in names}
    tokens = np.asarray(prob.inst.unit_tok)
    tokens = sorted({int(t) for t in np.quantile(tokens[tokens > 0], (0.0, 0.25, 0.5, 0.75, 1.0))})
    ok = all([run_block(s, tokens[len(tokens) // 2], a.tp) for s in specs.values()])

    samples = calibrate.measure([(s.hidden, s.ffn) for s in specs.values()], tokens, a.tp)
    base = np.tile([1 / MI355X["flops"], 1 / MI355X["mem_bw"], 1 / MI355X["net_bw"]], (N_KINDS, 1))
    coef = calibrate.fit(samples, base)
    for kind, name in ((calibrate.K_GEMM, "GEMM"), (calibrate.K_ELEM, "element-wise")):
        print(f"{name}: {1 / coef[kind, 0] / 1e12:.0f} TFLOP/s, {1 / coef[kind, 1] / 1e12:.2f} TB/s")
    print(f"accuracy on the samples: {calibrate.accuracy(samples, base):.1%} before, "
          f"{calibrate.accuracy(samples, coef):.1%} after")

    table = dip.DeviceOpTable(operator_table(prob, a.tp), N_KINDS)
    out = torch.empty((1, table.n_items), dtype=torch.int32, device="cuda")
    dip.cost_tables(table, torch.from_numpy(coef[None].copy()).cuda(), out)
    costs = out[0].cpu().numpy()
    prob = dataclasses.replace(prob, op_cost=costs[:prob.n_total], edge_comm=costs[prob.n_total:])
    orders = torch.from_numpy(np.ascontiguousarray(
        W.generator_for(prob, a.workload).generate(0, a.candidates))).cuda()
    sim = dip.Sim(prob)
    ms, _, _, flags = sim.evaluate(orders)
    index, best = dip.decode_key(int(sim.argmin(ms, flags).item()))
    good = ms[flags == 0]
    print(f"{a.candidates} schedules: best {best} us (candidate {index}), "
          f"mean {good.double().mean().item():.0f} us")
    return 0 if ok else 1


if __name__ == "__main__":
    sys.exit(main())

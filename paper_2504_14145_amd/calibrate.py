"""Coefficients of the cost tables from times on this card (DIP, arXiv
2504.14145, Sec. 6.1 and 7.4).

A row of an operator table costs max(c_fop N_fop, c_mem N_mem, c_net N_net)
seconds, with coefficients per kind of operator.  ``measure`` times the stage
operators -- matrix products with their epilogues, and layer norms -- forward and
backward, at token counts of a workload; ``fit`` turns such times into the
coefficients of their kinds, and ``cost_tables`` takes them.  Counts follow the
operator tables: 2-byte activations and weights, a backward twice its forward.
Kinds that are not measured (attention, collectives, transfers) keep what they
are given.
"""
from __future__ import annotations

from dataclasses import dataclass

import numpy as np

from . import ops

K_GEMM, K_ELEM = 0, 2     # kinds of the operator tables


@dataclass(frozen=True)
class Sample:
    kind: int
    n_fop: float
    n_mem: float
    seconds: float
    name: str


CALLS = 10                # timed in a row
APART = 1 << 29           # bytes between two uses of an array: twice the memory-side cache


def _time(run, sets, repeats: int) -> float:
    """Median seconds of a call of ``run`` among others on the current stream, each on
    the next of ``sets`` of arrays, none of which the caches hold."""
    import torch
    run(sets[0])
    run(sets[-1])
    other = torch.empty(APART, dtype=torch.uint8, device=sets[0][0].device)
    times = []
    for _ in range(repeats):
        other.zero_()
        a, b = (torch.cuda.Event(enable_timing=True) for _ in range(2))
        a.record()
        for i in range(CALLS):
            run(sets[i % len(sets)])
        b.record()
        b.synchronize()
        times.append(a.elapsed_time(b) * 1e-3 / CALLS)
    return sorted(times)[len(times) // 2]


def measure(modules, tokens, tp: int = 4, p: float = 0.1, repeats: int = 7, dtype=None,
            device="cuda") -> list:
    """Samples of every module (hidden, ffn) at every token count: the MLP's two
    products, one with the activation and one with dropout and the residual in
    its epilogue, and the layer norm, forward and backward, on arrays from memory."""
    import torch
    dtype = torch.bfloat16 if dtype is None else dtype
    out = []
    drop = ops.Dropout(p, 1) if p else None
    for h, f in modules:
        f = f // tp
        gamma, beta = (torch.empty(h, dtype=dtype, device=device).normal_(0, 0.02) for _ in range(2))
        for t in tokens:
            sets = []
            for _ in range(min(CALLS, -(-APART // (t * min(h, f) * gamma.element_size())))):
                x, u = (torch.empty((t, c), dtype=dtype, device=device).normal_() for c in (h, f))
                w1, w2 = (torch.empty(s, dtype=dtype, device=device).normal_(0, 0.02) for s in ((f, h), (h, f)))
                sets.append((x, u, torch.empty_like(u), w1, w2, x.unsqueeze(1)))
            calls = (
                ("MLP in", lambda a: ops.linear(a[0], a[3], act="gelu", pre=a[2]),
                 lambda a: ops.linear_backward(a[1], a[0], a[3], act="gelu", pre=a[2], bias=False)),
                ("MLP out", lambda a: ops.linear(a[1], a[4], dropout=drop, residual=a[0]),
                 lambda a: ops.linear_backward(a[0], a[1], a[4], dropout=drop, bias=False)))
            fop, mem = 2.0 * t * h * f, 2.0 * (t * h + h * f + t * f)
            for name, forward, backward in calls:
                for a in sets:
                    forward(a)
                out.append(Sample(K_GEMM, fop, mem, _time(forward, sets, repeats), f"{name} {t} x {h} x {f}"))
                out.append(Sample(K_GEMM, 2 * fop, 2 * mem, _time(backward, sets, repeats),
                                  f"{name} {t} x {h} x {f} backward"))
            _, mean, rstd = ops.group_norm(sets[0][5], 1, gamma, beta)
            fop, mem = 8.0 * t * h, 4.0 * t * h
            out.append(Sample(K_ELEM, fop, mem, _time(lambda a: ops.group_norm(a[5], 1, gamma, beta), sets, repeats),
                              f"layer norm {t} x {h}"))
            out.append(Sample(K_ELEM, 2 * fop, 2 * mem, _time(
                lambda a: ops.group_norm_backward(a[5], a[5], mean, rstd, 1, gamma, beta), sets, repeats),
                f"layer norm {t} x {h} backward"))
    return out


def predict(samples, coef) -> np.ndarray:
    """Seconds that the coefficients [kinds][3] give each sample."""
    c = np.asarray(coef, np.float64)
    return np.array([max(c[s.kind][0] * s.n_fop, c[s.kind][1] * s.n_mem) for s in samples])


def fit(samples, base) -> np.ndarray:
    """``base`` [kinds][3] (seconds per FLOP, per byte, per byte sent) with c_fop
    and c_mem of the measured kinds replaced.

    A sample's time is put down to the resource that the coefficients make the
    larger, starting with those of ``base``; each coefficient is the time of its
    samples over their count, so that long operators, which a schedule's length
    is made of, weigh most; and this is repeated until no sample changes sides.
    A resource without samples takes the least time per count: no sample can
    have a larger coefficient of it."""
    coef = np.array(base, np.float64)
    for kind in sorted({s.kind for s in samples}):
        rows = [s for s in samples if s.kind == kind]
        t = np.array([s.seconds for s in rows])
        n = np.array([[s.n_fop, s.n_mem] for s in rows])
        if not (t > 0).all() or not (n > 0).all():
            raise ValueError("a sample needs a time and counts above zero")
        side = (n * coef[kind, :2]).argmax(1)
        for _ in range(100):
            c = np.array([t[side == r].sum() / n[side == r, r].sum() if (side == r).any()
                          else (t / n[:, r]).min() for r in range(2)])
            new = (n * c).argmax(1)
            if (new == side).all():
                break
            side = new
        coef[kind, :2] = c
    return coef


def accuracy(samples, coef) -> float:
    """1 - the sum of the errors of the predicted times over the sum of the times."""
    t = np.array([s.seconds for s in samples])
    return float(1 - np.abs(predict(samples, coef) - t).sum() / t.sum())

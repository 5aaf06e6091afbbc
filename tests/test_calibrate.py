"""Fitting the cost tables' coefficients to times, on the CPU."""
import numpy as np
import pytest

from paper_2504_14145_amd.calibrate import K_ELEM, K_GEMM, Sample, accuracy, fit, predict
from workloads.operators import LLAMA3_8B, N_KINDS, layer_ops

BASE = np.tile([1e-15, 1e-13, 1e-11], (N_KINDS, 1))


def samples(c, noise=0.0, seed=0):
    rng = np.random.default_rng(seed)
    out = []
    for t in (1, 16, 200, 1500, 8192):
        for kind, fop, mem, _ in layer_ops(LLAMA3_8B, t, 4):
            if kind in (K_GEMM, K_ELEM):
                s = max(c[kind][0] * fop, c[kind][1] * mem) * float(np.exp(noise * rng.standard_normal()))
                out.append(Sample(kind, float(fop), float(mem), s, f"{t}"))
    return out


def test_recovers_planted_coefficients():
    c = BASE.copy()
    c[K_GEMM] = [1 / 1.2e15, 1 / 4.5e12, 7.0]
    c[K_ELEM] = [1e-20, 1 / 4.0e12, 7.0]
    s = samples(c)
    got = fit(s, BASE)
    assert np.allclose(predict(s, got), [x.seconds for x in s], rtol=1e-9)
    assert np.allclose(got[K_GEMM, :2], c[K_GEMM, :2], rtol=1e-9)
    assert np.isclose(got[K_ELEM, 1], c[K_ELEM, 1], rtol=1e-9)
    assert accuracy(s, got) > 1 - 1e-9


def test_other_kinds_and_the_network_keep_what_they_have():
    got = fit(samples(BASE), BASE)
    for kind in range(N_KINDS):
        if kind not in (K_GEMM, K_ELEM):
            assert np.array_equal(got[kind], BASE[kind])
    assert np.array_equal(got[:, 2], BASE[:, 2])


def test_noise_is_averaged():
    c = BASE.copy()
    c[K_GEMM, :2] = [1 / 1.2e15, 1 / 4.5e12]
    c[K_ELEM, :2] = [1e-20, 1 / 4e12]
    s = samples(c, noise=0.05, seed=3)
    got = fit(s, BASE)
    # 8 to 20 samples a coefficient: their mean is within 4 x 5 % / sqrt(8)
    assert abs(np.log(got[K_GEMM, 0] / c[K_GEMM, 0])) < 0.08
    assert abs(np.log(got[K_ELEM, 1] / c[K_ELEM, 1])) < 0.08
    assert accuracy(s, got) > 0.9


def test_refuses_times_that_are_none():
    with pytest.raises(ValueError):
        fit([Sample(K_GEMM, 1.0, 1.0, 0.0, "")], BASE)

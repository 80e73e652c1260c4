"""Iteration times as whole numbers: what rounding loses is found, said and avoided."""
import warnings

import numpy as np
import pytest

from paper_2608_16336_gb300 import workloads

torch = pytest.importorskip("torch")
from paper_2608_16336_gb300 import instance, mtsim  # noqa: E402

PAIRS = [(p, d) for p in (0, 256, 1024, 4096) for d in (0, 8, 32, 63) if p or d]


def made(base, a, b):
    return [(p, d, base + a * p + b * d) for p, d in PAIRS]


@pytest.mark.parametrize("base,a,b,per_us", [(300, 0.12, 0.4, 100), (2500, 1.4, 6.4, 10), (4000, 20, 30, 1), (90, 0.05, 0, 20)])
def test_finer_units_hold_the_model(base, a, b, per_us):
    with warnings.catch_warnings():
        warnings.simplefilter("error")
        times = instance.fit_iteration_times(made(base, a, b), per_us=per_us)
    assert times == (round(base * per_us), round(a * per_us), round(b * per_us))


def least(samples, bases, most):
    """The smallest sum of squares of any whole constants."""
    p, d, t = (np.array(v, dtype=float) for v in zip(*samples))
    base = np.arange(1, bases)[:, None]
    return min(float((((base + a * p + b * d) / t - 1) ** 2).sum(1).min()) for a in range(most) for b in range(most))


def off(samples, x):
    return sum(((x[0] + x[1] * p + x[2] * d) / t - 1) ** 2 for p, d, t in samples)


@pytest.mark.parametrize("base,a,b", [(300, 0.12, 0.4), (2500, 1.4, 6.4)])
def test_whole_microseconds_that_lose_are_reported_and_fitted_together(base, a, b):
    samples = made(base, a, b)
    with pytest.warns(RuntimeWarning, match="per_us"):
        times = instance.fit_iteration_times(samples)
    assert off(samples, times) <= least(samples, 6000, 12) * (1 + 1e-9)
    assert off(samples, times) < off(samples, (base, round(a), round(b)))  # each rounded by itself


def test_the_best_whole_numbers_are_found():
    g = np.random.default_rng(5)
    for _ in range(20):
        base, a, b = g.uniform(20, 60), g.uniform(0, 3), g.uniform(0, 3)
        samples = [(p, d, (base + a * p + b * d) * g.uniform(0.9, 1.1)) for p in (0, 3, 9, 20) for d in (0, 2, 7) if p or d]
        with warnings.catch_warnings():
            warnings.simplefilter("ignore")
            times = instance.fit_iteration_times(samples)
        assert off(samples, times) <= least(samples, 100, 8) * (1 + 1e-9), times


def test_a_workload_in_finer_units():
    w = workloads.config(0, requests=50)
    v = instance.with_times(w, (30000, 12, 40), per_us=100)
    assert (v.iter_base_us, v.iter_us_per_prefill_token, v.iter_us_per_decode_seq) == (30000, 12, 40)
    assert v.migrate_interval_us == 100 * w.migrate_interval_us and v.arrival_us.dtype == w.arrival_us.dtype
    assert np.array_equal(v.arrival_us, w.arrival_us * np.uint32(100))
    drained = instance.with_times(w, (1, 1, 1))
    drained.drain_start_us = np.array([[5, 0xFFFFFFFF]], np.uint32)
    assert instance.with_times(drained, (1, 1, 1), per_us=10).drain_start_us.tolist() == [[50, 0xFFFFFFFF]]
    late = instance.with_times(w, (1, 1, 1))
    late.arrival_us = np.array([429496730], np.uint32)
    with pytest.raises(ValueError, match="32 bits"):
        instance.with_times(late, (1, 1, 1), per_us=10)
    for bad in (0, 1.5):
        with pytest.raises(ValueError):
            instance.with_times(w, (1, 1, 1), per_us=bad)
        with pytest.raises(ValueError):
            instance.fit_iteration_times(made(1, 1, 1), per_us=bad)


@pytest.mark.gpu
def test_a_simulation_in_finer_units_is_the_same_simulation():
    """Ten times every time of a workload: ten times every time of its results."""
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    torch.cuda.set_device(0)
    w = workloads.config(0, requests=300)
    got = []
    for per_us in (1, 10):
        sim = mtsim.Simulator(instance.with_times(w, (4000 * per_us, 20 * per_us, 30 * per_us), per_us=per_us))
        sim.load()
        assert sim.run() == 0
        got.append(sim.metrics()[0])
        sim.close()
    for field in ("first_token_us", "finish_us"):
        a, b = (r[field].astype(np.int64) for r in got)
        assert np.array_equal(a * 10, b) and (a < 0xFFFFFFFF).all()

"""The probe's intervals hold what a cell can do at any times between the fast
and the slow ones, across the loads at which another batch is taken (no GPU
needed)."""
import random

import numpy as np
import pytest

from paper_2608_19659_amd import probe
from paper_2608_19659_amd.synth import Problem


def between(pair, share):
    return pair[0] + share * (pair[1] - pair[0])


def test_a_switch_of_batches_between_the_two_sides():
    """At the fast times a batch of 1 serves the load with a rate of 1, at the
    slow ones a batch of 4 with 1.176; between them rates go from the load to 1.379."""
    load, prefill, steps = 0.95, (0.1, 0.1), {1: (0.009, 0.012), 4: (0.020, 0.030)}
    cap, tail = probe.settle_between(load, 100, prefill, steps)
    assert probe.settle(load, 100, 0.1, {1: 0.0105, 4: 0.025})[0] == pytest.approx(1 / 0.725)
    assert cap[0] == pytest.approx(0.95) and cap[1] == pytest.approx(1 / 0.6)
    assert tail[0] == pytest.approx(1.0 / 0.905) and tail[1] == pytest.approx(3.1 / 0.905)
    # no batch serves it at the slow times
    cap, tail = probe.settle_between(1.5, 100, prefill, steps)
    assert cap == (pytest.approx(1 / 0.85), pytest.approx(1 / 0.6)) and tail == (pytest.approx(2.1 / 0.85), probe.UNSERVED)
    # nor at the fast ones
    cap, tail = probe.settle_between(5.0, 100, prefill, steps)
    assert cap == (pytest.approx(1 / 0.85), pytest.approx(1 / 0.6)) and tail == (probe.UNSERVED, probe.UNSERVED)


@pytest.mark.parametrize("seed", range(40))
def test_all_times_between_the_sides(seed):
    r = random.Random(seed)
    classes = (probe.Class("a", 10, r.choice([1, 20, 100]), 4.0, 5.0),)
    levels = sorted({round(2.0 ** r.uniform(-3, 3), 3) for _ in range(6)})
    problem = Problem(tp=[1], levels=levels, demand=[4.0], slo=[5.0], budget=8)
    pair = lambda x: (x, x * r.uniform(1.0, 2.0))  # noqa: E731
    times = probe.Times()
    prefill = times.prefill[1, "a"] = pair(r.uniform(0.02, 0.5))
    base = 2.0 / classes[0].answer * r.uniform(0.1, 1.0)
    steps = times.step[1, "a"] = {n: pair(base * n ** r.uniform(0.2, 0.9)) for n in (1, 2, 4, 16, 64)}
    iv = probe.intervals(problem, classes, times)
    for cell in range(problem.n_cells):
        load = float(problem.levels[problem.cell_coords(cell)[2]])
        for _ in range(300):
            ends = r.random() < 0.3
            share = lambda: r.choice([0.0, 1.0]) if ends else r.random()  # noqa: E731
            cap, tail = probe.settle(load, classes[0].answer, between(prefill, share()), {n: between(s, share()) for n, s in steps.items()})
            assert iv.cap_lo[0, cell] <= cap <= iv.cap_hi[0, cell]
            assert iv.tail_lo[0, cell] <= np.float32(tail) <= iv.tail_hi[0, cell]

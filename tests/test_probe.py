"""The probe's arithmetic: from times to cells (no GPU needed)."""
import numpy as np
import pytest

from paper_2608_19659_amd import probe
from paper_2608_19659_amd.synth import Problem


def test_the_smallest_batch_that_serves_the_load():
    steps = {1: 0.010, 4: 0.016, 16: 0.032}
    # a batch of 1: 1 / (0.1 + 100 * 0.010) = 1 / 1.1; of 4: 1 / (0.1 + 0.4); of 16: 1 / (0.1 + 0.2)
    rate, tail = probe.settle(0.5, 100, 0.1, steps)
    assert rate == pytest.approx(1 / 1.1) and tail == pytest.approx(1.1 / 0.95)
    rate, tail = probe.settle(2.0, 100, 0.1, steps)
    assert rate == pytest.approx(2.0) and tail == pytest.approx(1.7 / 0.8)
    rate, tail = probe.settle(3.0, 100, 0.1, steps)
    assert rate == pytest.approx(1 / 0.3) and tail == pytest.approx(3.3 / 0.7)
    rate, tail = probe.settle(4.0, 100, 0.1, steps)
    assert rate == pytest.approx(1 / 0.3) and tail == probe.UNSERVED


def test_the_sum_over_ranks():
    d = probe.Decoder(hidden=1000, layers=10)
    assert probe.sum_seconds(d, 1, 5, 100.0, 1.0) == 0.0
    # 20 sums of 2 * 3/4 * 5 * 1000 * 2 bytes at 100 GB/s and 6 hops of 1 us
    assert probe.sum_seconds(d, 4, 5, 100.0, 1.0) == pytest.approx(20 * (15000 / 100e9 + 6e-6))


def test_intervals_hold_both_sides_on_the_grid():
    classes = (probe.Class("a", 10, 100, 4.0, 5.0), probe.Class("b", 10, 20, 2.0, 5.0))
    problem = Problem(tp=[1, 2], levels=[0.5, 2.0, 8.0], demand=[4.0, 2.0], slo=[5.0, 5.0], budget=8)
    times = probe.Times()
    for tp in (1, 2):
        for c in classes:
            times.prefill[tp, c.name] = (0.05 / tp, 0.06 / tp)
            times.step[tp, c.name] = {1: (0.01 / tp, 0.012 / tp), 8: (0.02 / tp, 0.021 / tp)}
    iv = probe.intervals(problem, classes, times)
    assert iv.cap_lo.shape == (1, problem.n_cells) and iv.cap_lo.dtype == np.float32
    assert not iv.measured.any()
    assert (iv.cap_lo > 0).all() and (iv.cap_hi >= iv.cap_lo).all() and (iv.tail_hi >= iv.tail_lo).all()
    assert np.isfinite(iv.tail_hi).all()
    for x in (iv.cap_lo, iv.cap_hi):
        assert (x * 64 == np.rint(x * 64)).all()
    for cell in range(problem.n_cells):
        i, t, b = problem.cell_coords(cell)
        key = int(problem.tp[t]), classes[i].name
        for side in (0, 1):
            cap, tail = probe.settle(float(problem.levels[b]), classes[i].answer, times.prefill[key][side],
                                     {n: s[side] for n, s in times.step[key].items()})
            assert iv.cap_lo[0, cell] <= cap <= iv.cap_hi[0, cell]
            assert iv.tail_lo[0, cell] <= np.float32(tail) <= iv.tail_hi[0, cell]


@pytest.mark.parametrize("argv", [["--tp", "3"], ["--tp", "16"], ["--batch", "0"], ["--layers", "0"], ["--budget", "0"],
                                  ["--batch", "5000"], ["--link-gbs", "0"]], ids=" ".join)
def test_arguments_that_are_refused(argv, capsys):
    with pytest.raises(SystemExit) as e:
        probe.main(argv)
    assert e.value.code == 2

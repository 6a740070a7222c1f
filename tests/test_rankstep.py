"""A rank's step and the trace of a job whose ranks take it: what needs no GPU."""
import numpy as np
import pytest

from oracle import ccld_oracle as orc
from paper_2605_04478_amd import rankstep, tracegen as tg


def test_even_load():
    assert rankstep.even_load(10, 4) == [2, 3, 2, 3] and sum(rankstep.even_load(4097, 8)) == 4097
    assert rankstep.even_load(0, 3) == [0, 0, 0]


@pytest.mark.parametrize("busy", [0, 5, 15])
def test_the_rank_that_computes_longer_is_named(busy):
    compute = np.full(16, 2_000_000, dtype=np.int64)
    compute[busy] = 3_500_000
    tr = rankstep.trace(compute, n_slots=60)
    assert tr.n == 60 * 16 and len(tr.topo.size) == tg.Layout3D(tp=16, pp=1, dp=1).topology().n_comms
    o = orc.Oracle(tr.topo).analyze_window(tr.cols, int(tr.cols["t_exit"].max()) + 1)
    assert int(o.order[0]) == busy
    assert int(o.blame["n_late_enter"][busy]) >= 59 and int(np.delete(o.blame["n_late_enter"], busy).sum()) == 0


def test_equal_ranks_raise_no_flag():
    tr = rankstep.trace(np.full(8, 2_000_000, dtype=np.int64), n_slots=40)
    o = orc.Oracle(tr.topo).analyze_window(tr.cols, int(tr.cols["t_exit"].max()) + 1)
    assert not o.blame["n_late_enter"].any()


def test_one_gap_for_all_is_the_same_as_one_each():
    tr = tg.generate(tg.config1(n_slots=30, faults=False))
    a, b = tg.propagate(tr, 1_000_000), tg.propagate(tr, np.full(16, 1_000_000, dtype=np.int64))
    assert all(np.array_equal(a.cols[k], b.cols[k]) for k in a.cols)

"""The cut of adsa_shared_prefix_attn's work, on the host: runs follow each other without a gap, none is empty while there are
units, and the run that the merge finds for a unit is the one that holds it."""
import numpy as np
import pytest

from prefix_cut import Cut, WideCut


def totals(resident):
    edges = {0, 1, 2, 3, resident - 1, resident, resident + 1, 2 * resident + 7, 10**6 + 3, 4 * 10**6}
    for fours in range(1, 20):                                    # every border between numbers of sizes, and around the pieces
        for d in (-resident, -1, 0, 1, 2, resident // 3, resident + 1):
            edges.add(max(0, 4 * fours * resident + d))
    rng = np.random.default_rng(resident)
    return sorted(edges | set(rng.integers(0, 40 * 4 * resident, 60).tolist()))


def check(cut, total, most_runs):
    assert cut.runs <= most_runs
    if total == 0:
        return
    begin = cut.begin_of(np.arange(cut.runs + 1))
    assert begin[0] == 0 and begin[-1] == total and (np.diff(begin) > 0).all()
    holds = np.repeat(np.arange(cut.runs), np.diff(begin))
    assert (cut.run_of(np.arange(total)) == holds).all()


@pytest.mark.parametrize("resident", [1, 2, 5, 74, 132, 148, 264, 296])
def test_runs_of_the_sweep(resident):
    seen = set()
    for total in totals(resident):
        cut = Cut(total, resident)
        seen.add(cut.K)
        check(cut, total, 5 * resident)
    assert seen == {1, 2, 3, 4, 5}


@pytest.mark.parametrize("resident", [1, 2, 74, 148])
def test_runs_of_the_wide_kernel(resident):
    for total in totals(resident):
        cut = WideCut(total, resident)
        check(cut, total, resident)
        if total >= 2:
            assert (np.diff(cut.begin_of(np.arange(cut.runs + 1))) >= 2).all()

"""CPU: tables of frequencies that are no numbers are refused."""
import numpy as np
import pytest

from paper_2602_07529_amd import binding as B

INF = float("inf")


@pytest.mark.parametrize("args", [(1e4, 4.0, 8192.0, -INF, 32.0), (1e4, 4.0, 8192.0, -INF, INF), (1e4, 1e-320, 8192.0, 1.0, 4.0), (1e4, 1e-320, 0.0, 1.0, 4.0),
                                  (1e-300, 1e-300, 0.0, 1.0, 4.0)])
def test_refused(args):
    freq = np.full(32, 7.0)
    assert B.lib().dag_rope_frequencies(freq.ctypes.data, 64, *args) == -7
    assert (freq == 7.0).all()
    with pytest.raises(B.DagError):
        B.Rope(64, args[0], "cpu", stretch=args[1], original=args[2], low=args[3], high=args[4])


def test_a_pair_that_turns_ever_so_often():
    """high = infinity: no pair turns that often, all are interpolated."""
    freq, all_of_them = np.empty(32), np.empty(32)
    assert B.lib().dag_rope_frequencies(freq.ctypes.data, 64, 1e4, 4.0, 8192.0, 1.0, INF) == 0
    assert B.lib().dag_rope_frequencies(all_of_them.ctypes.data, 64, 1e4, 4.0, 0.0, 1.0, 32.0) == 0
    assert np.array_equal(freq, all_of_them)

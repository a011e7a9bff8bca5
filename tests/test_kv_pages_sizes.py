"""CPU: numbers of rows and forks that the calls on shared pages cannot count are refused."""
import ctypes as C

import pytest

from paper_2602_07529_amd import binding as B
from tests.test_q8_more_refusals import COMPACT, FAKE, FORK, RELEASE


@pytest.mark.parametrize("n", [2 ** 27, 2 ** 31 - 1000, 2 ** 31 - 1])
def test_rows_and_forks_past_32_bits(n):
    lib, huge = B.lib(), 2 ** 62
    rows = lambda n: C.byref(B.dag_kv_rows_t(n, 16, 1, 50, FAKE, FAKE))  # noqa: E731
    assert lib.dag_kv_fork(rows(n), *FORK, FAKE, huge, None) == -2
    assert lib.dag_kv_fork(rows(4), n, *FORK[1:], FAKE, huge, None) == -2
    assert lib.dag_kv_release_shared(rows(n), *RELEASE, FAKE, huge, None) == -2
    assert lib.dag_kv_compact(rows(n), rows(n), *COMPACT, FAKE, huge, None) == -2

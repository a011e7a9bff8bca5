"""Calls on shared pages with as many forks, rows and pages as take other paths than small ones, or more workgroups than a launch."""
import numpy as np
import pytest
import torch

from paper_2602_07529_amd import binding as B
from tests.gpu_util import DEV
from tests.q8_cases import ints
from tests.test_gpu_kv_pages import Family

pytestmark = pytest.mark.gpu


def test_forks_past_the_threads_of_a_launch():
    """2^24 entries and some: all but three ask for children that are taken, and are refused."""
    n = (1 << 24) + 77
    f = Family([50, 0, 33, 0, 0], 4, 30, seed=9)
    parent, child = (torch.zeros(n, dtype=torch.int32, device=DEV) for _ in range(2))
    child.fill_(2)  # (holds tokens)
    at = [1, 1 << 23, n - 1]
    parent[at], child[at] = ints([2, 0, 2]), ints([1, 3, 4])
    src, dst, refused = (torch.zeros(m, dtype=torch.int32, device=DEV) for m in (n, n, 1))
    before = f.rows.table.clone()
    B.dag_kv_fork(f.rows, parent, child, f.d_len, f.d_len, f.d_extra, f.d_extra, f.d_count, f.d_count, src, dst, refused=refused)
    assert int(refused) == n - 3 and f.d_len.tolist() == [50, 33, 33, 50, 33] and int(f.d_count) == f.count - 3
    some = torch.nonzero(src >= 0)[:, 0].tolist()
    free = f.free[:f.count]
    assert some == at and src[at].tolist() == [int(before[2, 2]), int(before[0, 3]), int(before[2, 2])] and dst[at].tolist() == free[::-1][:3].tolist()
    table = f.rows.table
    for i, (p, c, full) in enumerate(((2, 1, 2), (0, 3, 3), (2, 4, 2))):
        assert torch.equal(table[c, :full], before[p, :full]) and int(table[c, full]) == int(dst[at[i]])
    holders = np.zeros(len(f.extra), dtype=np.int64)
    np.add.at(holders, before[0, :3].cpu().numpy(), 1)
    np.add.at(holders, before[2, :2].cpu().numpy(), 2)
    assert np.array_equal(f.d_extra.cpu().numpy(), holders)


@pytest.mark.parametrize("in_place", [True, False])
def test_pools_whose_bitmap_does_not_fit_lds(in_place):
    """More than 262144 pages, not a multiple of the 32 of a word."""
    f = Family([900 * 16 - 5] * 150 + [0] * 9, 900, 262181 - 150 * 900, seed=11)
    f.fork([3] * 4 + [7] * 5, list(range(150, 159)), [0, 17, 5000, 10 ** 5, 16, 1, 15, 14000, 48], in_place)
    for _ in range(2):
        assert len(f.compact(in_place)) in (0, *range(30000, 131072))
    f = Family([16] * 3 + [1], 2, 262145 + 31, seed=12)  # (nearly all free)
    f.compact(in_place)

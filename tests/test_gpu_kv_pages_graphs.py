"""Captured calls on shared pages beside eager ones of the same rows."""
import numpy as np
import pytest
import torch

from oracle import q8_oracle as q8
from paper_2602_07529_amd import binding as B
from tests.gpu_util import DEV
from tests.q8_cases import ints
from tests.test_gpu_kv_pages import Family

pytestmark = pytest.mark.gpu


def test_replays_behind_a_longer_list_of_forks():
    """The eager call needs a larger workspace; what the graph writes to stays the rows' own."""
    f = Family([50, 0, 33, 0, 0, 0], 8, 30, seed=7)
    parent, child, ended = [0, 0, 2], [1, 3, 4], [0, 1, 0, 1, 1, 1]
    src, dst, refused = ints([0] * 3), ints([0] * 3), ints([0])
    d_parent, d_child, d_ended = ints(parent), ints(child), ints(ended)
    size = f.rows.for_shared().numel()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        B.dag_kv_fork(f.rows, d_parent, d_child, f.d_len, f.d_len, f.d_extra, f.d_extra, f.d_count, f.d_count, src, dst, refused=refused)
        B.dag_kv_release_shared(f.rows, d_ended, f.d_len, f.d_len, f.d_extra, f.d_extra, f.d_count, f.d_count)
    many = [0] * 200
    f.fork(many, [5] * 200, [0] + [17] * 199)  # (padded: entries behind the first ask for the same child)
    others = [torch.full((size,), 0x5a, dtype=torch.uint8, device=DEV) for _ in range(64)]  # whoever asks for as much memory now
    for _ in range(3):
        graph.replay()
        torch.cuda.synchronize()
        f.count, s, d, bad = q8.fork(f.table, f.free, f.count, f.row_len, f.extra, parent, child, None)
        assert src.tolist() == list(s) and dst.tolist() == list(d) and int(refused) == bad
        f.count = q8.release_shared(f.table, f.free, f.count, f.row_len, f.extra, ended)
        f.same()
        f.fork(many, [5] * 200, [0] + [17] * 199)
        assert all(bool((x == 0x5a).all()) for x in others)
    assert np.array_equal(f.row_len, [50, 0, 33, 0, 0, 0])

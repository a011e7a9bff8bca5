"""CPU: the workspaces that a table of rows keeps for the calls on shared pages."""
import weakref

import torch

from paper_2602_07529_amd import binding as B


def rows_of(n, width, pages):
    return B.KvRows(torch.zeros((n, width), dtype=torch.int32), torch.zeros(pages, dtype=torch.int32))


def test_a_workspace_that_a_graph_may_hold_lives_as_long_as_the_rows():
    """A captured call has the address of the workspace: one with more forks than there are rows must not give that memory away."""
    rows = rows_of(4, 8, 50)
    first = weakref.ref(rows.for_shared())
    second = weakref.ref(rows.for_shared(100))
    assert rows.for_shared(4) is second() and rows.for_shared(100) is second()
    assert second().numel() >= B.lib().dag_kv_pages_workspace_bytes(4, 50, 100)
    rows.for_shared(1000)
    assert first() is not None and second() is not None
    del rows
    assert first() is None and second() is None


def test_lists_that_grow_take_few_workspaces():
    rows, held = rows_of(4, 8, 50), {}
    for n in range(1, 3000):
        ws = rows.for_shared(n)
        assert ws.numel() >= B.lib().dag_kv_pages_workspace_bytes(4, 50, n)
        held[ws.data_ptr()] = ws.numel()
    assert len(held) <= 12 and sum(held.values()) <= 2 * 4 * 2 * 3000 + 12 * 1000

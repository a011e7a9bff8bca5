"""CPU: what the drivers over the 8-bit cache refuse, before any GPU work."""
import pytest
import torch

from paper_2602_07529_amd import binding as B
from paper_2602_07529_amd import engine


def fork(n_pages, prefix, n_branches, max_len):
    k = torch.zeros((prefix, 2, 64), dtype=torch.bfloat16)
    return engine.Fork(B.KvCacheQ8.empty(n_pages, 2, 64, "cpu"), k, k, n_branches, max_len, 4, 1e4)


@pytest.mark.parametrize("n_pages,prefix,n_branches,max_len", [(2, 33, 0, 0), (2, 0, 3, 5), (5, 0, 3, 17), (6, 16, 3, 32), (7, 17, 3, 17)])
def test_a_cache_that_cannot_hold_the_prefix_and_its_branches(n_pages, prefix, n_branches, max_len):
    with pytest.raises(ValueError, match="pages"):
        fork(n_pages, prefix, n_branches, max_len)


def test_a_cache_that_just_holds_them():
    fork(6, 0, 3, 17)


def test_a_step_takes_a_token_of_every_branch():
    f = fork(6, 0, 3, 17)
    q, k = torch.zeros((3, 4, 64), dtype=torch.bfloat16), torch.zeros((3, 2, 64), dtype=torch.bfloat16)
    for bad in ((q[:1], k, k), (q, k[:1], k), (q, k, k[:, :1]), (q[0], k, k), (q[..., :1], k, k)):
        with pytest.raises(ValueError):
            f.step(*bad)
    assert f.tokens == 0

"""Scores of chunks are products of bf16 queries with codes that bf16 holds exactly: nothing of a query is lost beside a larger element of it."""
import pytest

import torch

from tests.q8_chunk_cases import Chunks

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("new", [3, 50])
@pytest.mark.parametrize("far", [2.0 ** 16, 2.0 ** 40])
def test_elements_of_a_query_far_apart(new, far):
    """The keys are zero in the dim of the large element, so it adds zeros, exactly: the bound is that of any call."""
    c = Chunks([([16] * 4 + [5], new, new)], 4, 1, 128, seed=22)
    c.q[:, :, 77] *= far
    codes = c.cache.k_pool.view(torch.uint8)
    codes[:, :, 4, :, 13] = 0
    c.call()
    c.check()

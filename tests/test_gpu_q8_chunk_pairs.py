"""Chunks whose nodes have numbers of (row, query head) pairs around those that change the kernel, its blocks or its cut: 32, 64, 96, 128 and 256."""
import numpy as np
import pytest

from tests.q8_chunk_cases import Chunks

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("hq,hkv,d", [(2, 2, 64), (8, 2, 128), (5, 1, 128)])
@pytest.mark.parametrize("pairs", [64, 65, 96, 97, 127, 128, 129, 255, 257])
def test_one_node(hq, hkv, d, pairs):
    new = -(-pairs // (hq // hkv))
    c = Chunks([([16] * 7 + [5], new + 4, new)], hq, hkv, d, seed=pairs, idle=2)
    c.call()
    c.check()


@pytest.mark.parametrize("hq,hkv,d", [(2, 2, 64), (8, 2, 128)])
@pytest.mark.parametrize("front", [3, 60])
def test_nodes_of_all_numbers_together(hq, hkv, d, front):
    g = hq // hkv
    news = [max(1, (p + e) // g) for p in (32, 64, 96, 128, 256) for e in (-g, 0, g)]
    c = Chunks([([16] * (front + i % 3) + [9], new + 7 * (i % 4), new) for i, new in enumerate(news)], hq, hkv, d, seed=front, idle=3, spare=5)
    c.call()
    rng, ends = np.random.default_rng(front), np.cumsum([0] + news)
    some = {int(x) for a, b in zip(ends, ends[1:]) for x in (a, b - 1, *rng.integers(a, b, 4))}
    c.check(rows=sorted(some))
    assert c.out[:c.n].isfinite().all()

"""GPU: appends of thousands of tokens to the 8-bit cache, whose workgroups take 4 or 16 tokens and the runs that start in them, against the
oracle (tolerances: test_gpu_q8_append)."""
import numpy as np
import pytest
import torch

from tests.test_gpu_q8_append import PAGE, Both, _new

pytestmark = pytest.mark.gpu


def _runs(rng, n, mix):
    """n slots in runs of lengths drawn from `mix`, each at the end of a page's tokens so far, some outside the pool; pages in any order.
    Returns the slots and what has to be in front of them."""
    slots, first, page = [], [], 0
    while len(slots) < n:
        left = min(int(rng.choice(mix)), n - len(slots))
        if rng.random() < 0.05:
            slots += [-1] * min(left, 3)
            continue
        i0 = 0 if rng.random() < 0.7 else int(rng.integers(0, PAGE))
        first += [page * PAGE + i for i in range(i0)]
        slots += [page * PAGE + i0 + i for i in range(left)]
        page += -(-(i0 + left) // PAGE)
    perm = rng.permutation(page + 1)
    there = lambda x: [int(perm[s // PAGE]) * PAGE + s % PAGE if s >= 0 else s for s in x]  # noqa: E731
    return there(slots), there(first), page + 1


MIXES = {"single": [1], "short": [1, 1, 2, 3, 5, 9], "any": [1, 4, 15, 16, 17, 33], "pages": [16, 32, 160], "long": [300, 2000]}


@pytest.mark.parametrize("n", [2047, 2048, 8191, 8192])
@pytest.mark.parametrize("mix", ["short", "any"])
@pytest.mark.parametrize("hkv,d,dtype", [(1, 64, torch.bfloat16), (1, 128, torch.float32)])
def test_counts_beside_the_borders_of_the_workgroups(n, mix, hkv, d, dtype):
    _append(n, mix, hkv, d, dtype)


@pytest.mark.parametrize("n", [2100, 9000])
@pytest.mark.parametrize("mix", list(MIXES))
@pytest.mark.parametrize("hkv,d,dtype", [(3, 128, torch.bfloat16), (2, 64, torch.float32)])
def test_runs_shared_out_over_the_waves_of_a_workgroup(n, mix, hkv, d, dtype):
    _append(n, mix, hkv, d, dtype)


@pytest.mark.parametrize("n", [2101, 8207])
@pytest.mark.parametrize("hkv,d,dtype", [(5, 64, torch.bfloat16), (8, 128, torch.float32)])
def test_more_heads_than_waves(n, hkv, d, dtype):
    _append(n, "any", hkv, d, dtype)


def _append(n, mix, hkv, d, dtype):
    rng = np.random.default_rng(n + hkv)
    slots, first, pages = _runs(rng, n, MIXES[mix])
    b = Both(pages, hkv, d, junk=False)
    if first:
        k, v = _new(n, len(first), hkv, d, dtype)
        b.append(first, np.arange(len(first)), k, v, 1e4)
    k, v = _new(n + 1, n, hkv, d, dtype, spread=1.0)
    b.append(slots, rng.integers(0, 100000, n), k, v, 5e5)


@pytest.mark.parametrize("n", [2500, 9001])
def test_many_tokens_give_the_bits_of_a_token_at_a_time(n):
    """Pages that begin: one call against calls of less than a workgroup's worth, run by run."""
    hkv, d = 3, 128
    k, v = _new(n, n, hkv, d, torch.bfloat16)
    pos = np.random.default_rng(n).integers(0, 5000, n)
    one, parts = Both(-(-n // PAGE), hkv, d, junk=False), Both(-(-n // PAGE), hkv, d, junk=False)
    one.append(np.arange(n), pos, k, v, 1e4)
    for a in range(0, n, 1600):
        parts.append(np.arange(a, min(n, a + 1600)), pos[a:a + 1600], k[a:a + 1600], v[a:a + 1600], 1e4)
    for x, y in ((one.cache.k_pool, parts.cache.k_pool), (one.cache.v_pool, parts.cache.v_pool), (one.cache.k_scale, parts.cache.k_scale)):
        assert torch.equal(x.view(torch.uint8), y.view(torch.uint8))

"""Tiny value scales of an 8-bit cache: a page of zeros has 2^-100.  They go into the exponent of the probabilities, whose results end at 2^-126, so
keys 2^-27 of the largest on such pages are where a sum of the probabilities could lose them.

Queries are (1, 0, ..), keys (16, 0, ..) or zero, so that a score is 16 or 0 times the softmax scale, exactly but for one rounding: FAR = 26.5 powers of
two apart, off by 28 * 2^-23 = 2^-18 at most."""
import math

import numpy as np
import pytest
import torch

from paper_2602_07529_amd import binding as B
from tests.gpu_util import DEV
from tests.q8_cases import ints

pytestmark = pytest.mark.gpu

FAR = 26.5
SCALE = FAR * math.log(2.0) / 16
ZEROS, TOP, SMALL, TOP_OF_SMALL = range(4)  # pages: zeros; a large key with a value; values of 256 * 2^-100; a large key without


def cache_of(d):
    cache = B.KvCacheQ8.empty(4, 1, d, DEV)
    k, v = cache.k_pool.view(torch.uint8), cache.v_pool.view(torch.uint8)
    k.zero_(), v.zero_()
    cache.k_scale.fill_(1.0)
    cache.v_scale.fill_(2.0 ** -100)
    cache.k_pool[TOP, 0, 0, 0, 0] = cache.k_pool[TOP_OF_SMALL, 0, 0, 0, 0] = 16.0
    value = torch.randn(d, generator=torch.Generator().manual_seed(1)).to(torch.float8_e4m3fn)
    v[TOP, 0, :, 0] = value.view(torch.uint8).to(DEV)
    cache.v_scale[TOP] = 1.0
    cache.v_pool[SMALL] = torch.full((1, d, 16), 256.0, device=DEV).to(torch.float8_e4m3fn)
    return cache, value.double()


def queries(n, hq, d):
    q = torch.zeros((n, hq, d), dtype=torch.bfloat16, device=DEV)
    q[:, :, 0] = 1.0
    return q


def chunk(cache, pages, new, hq, d):
    """One node whose last three pages are its own, full.  Output, log-sum-exp and the tokens that every row sees."""
    q = queries(new, hq, d)
    n = len(pages)
    desc = B.PagedPrefillDesc.on_device(1, new, n, ints([0, new]), ints([0, n]), ints(pages), ints([16] * n), ints([n - 3]), ints([48]))
    out, lse = torch.full_like(q, 7.0), torch.full((new, hq), 7.0, device=DEV)
    ws = torch.full((max(256, B.dag_prefill_paged_q8_workspace_bytes(desc, cache, new, hq)),), 0xff, dtype=torch.uint8, device=DEV)
    B.dag_attn_prefill_paged_q8(desc, q, cache, out, ws, lse=lse, softmax_scale=SCALE)
    return out.double().cpu(), lse.double().cpu(), 16 * n - new + 1 + np.arange(new)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("new", [1, 40])
@pytest.mark.parametrize("none", [False, True])
def test_chunk_counts_the_keys_of_pages_of_zeros(new, d, none):
    """2^20 keys, a large one among 2^14 each: 2^-12.5 of the sum is on the others.  Sums of up to 2^10 blocks a stretch, each rounded, 2^-24 at random signs
    or 2^-14 of a 2^-12.5 part at worst; the logarithm of 2^32, 22, is off by 2^-19 and its two terms by 2^-18: 2^-15 in all, half of the difference being 2^-13.5."""
    cache, value = cache_of(d)
    n, hq = 1 << 16, 4
    pages = np.full(n, ZEROS)
    pages[::1 << 10] = TOP
    if none:  # a value that is no number, in one dim: the sums are taken once more
        cache.v_pool.view(torch.uint8)[ZEROS, 0, 7, 4] = 0x7f
    out, lse, seen = chunk(cache, pages, new, hq, d)
    tops = len(pages[::1 << 10])
    weight = 2.0 ** FAR * tops
    total = weight + seen - tops
    assert (np.abs(lse.numpy() - np.log(total)[:, None]) <= 2.0 ** -15).all()
    want = value * torch.from_numpy(weight / total)[:, None, None]
    if none:
        assert out[:, :, 7].isnan().all()
        out[:, :, 7] = want[:, :, 7]
    assert ((out - want).abs() <= want.abs() * (2.0 ** -8 + 2.0 ** -14)).all()


def small(n):
    """A large key without a value in front of n pages of tiny values."""
    return np.array([TOP_OF_SMALL] + [SMALL] * n)


def of_small(seen):
    """What comes out: the first page has one large key and 15 others, none of them with a value."""
    return 256.0 * 2.0 ** -100 * (seen - 16) / (2.0 ** FAR + seen - 1)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("new", [1, 40])
@pytest.mark.parametrize("none", [False, True])
def test_chunk_over_tiny_values(new, d, none):
    """Probabilities and result are rounded to bf16 (2^-8 each, all of one probability the same way), scores are off by 2^-18."""
    cache, _ = cache_of(d)
    if none:
        cache.v_pool.view(torch.uint8)[SMALL, 0, 7, 4] = 0xff
    out, lse, seen = chunk(cache, small(9), new, 4, d)
    want = torch.from_numpy(of_small(seen))[:, None, None].expand(out.shape)
    if none:
        assert out[:, :, 7].isnan().all()
        out[:, :, 7] = want[:, :, 7]
    assert ((out - want).abs() <= want * (2 * 2.0 ** -8 + 2.0 ** -15)).all()

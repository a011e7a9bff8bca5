"""Tiny value scales of an 8-bit cache: a page of zeros has 2^-100.  They go into the exponent of the probabilities, whose results end at 2^-126, so
keys 2^-27 of the largest on such pages are where a sum of the probabilities could lose them.

Queries are (1, 0, ..), keys (16, 0, ..), zero or (-448, 0, ..), so that a score is 16, 0 or -448 times the softmax scale, exactly but for one
rounding: the first two are FAR = 26.5 powers of two apart, off by 2^-18 at most, the third does not count.  Lists of pages alternate: zeros at even
places, a large key or nothing at odd ones, as a lane adds up every other page: so the sum of the zeros does not start from that of a large key, which
would round every block's part of it.  They are added up a block after the other, n equal parts rounded to n 2^-24 of their sum at most."""
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
# pages: zeros; a large key with a value, and keys that do not count; such keys only; values of 256 * 2^-100; a large key without a value
ZEROS, TOP, NOTHING, SMALL, TOP_OF_SMALL = range(5)


def cache_of(d, value=1.5, scale=1.0):
    cache = B.KvCacheQ8.empty(5, 1, d, DEV)
    cache.k_pool.view(torch.uint8).zero_()
    cache.v_pool.view(torch.uint8).zero_()
    cache.k_scale.fill_(1.0)
    cache.v_scale.fill_(2.0 ** -100)
    for page in (TOP, NOTHING, TOP_OF_SMALL):
        cache.k_pool[page, 0, 0, :, 0] = torch.full((16,), -448.0, device=DEV).to(torch.float8_e4m3fn)
    cache.k_pool[TOP, 0, 0, 0, 0] = cache.k_pool[TOP_OF_SMALL, 0, 0, 0, 0] = 16.0
    cache.v_pool[TOP, 0, :, 0] = torch.full((d,), value, device=DEV).to(torch.float8_e4m3fn)
    cache.v_scale[TOP] = scale
    cache.v_pool[SMALL] = torch.full((1, d, 16), 256.0, device=DEV).to(torch.float8_e4m3fn)
    return cache


def queries(n, hq, d):
    q = torch.zeros((n, hq, d), dtype=torch.bfloat16, device=DEV)
    q[:, :, 0] = 1.0
    return q


def pages_of(n, even, top, period):
    pages = np.tile(np.array([even, NOTHING], dtype=np.int32), n // 2)
    pages[1::period] = top
    return pages


def counts(pages, even, seen):
    """Large keys, and tokens on pages `even`, among the first `seen` tokens (all on the last page are of the latter or do not count)."""
    whole = seen // 16
    tops = np.isin(pages[:whole], (TOP, TOP_OF_SMALL)).sum()
    return tops, 16 * (pages[:whole] == even).sum() + (seen % 16 if seen % 16 and pages[whole] == even else 0)


def chunk(cache, pages, new, hq, d):
    """One node whose last three pages are its own, full.  Output, log-sum-exp and the tokens that every row sees."""
    q = queries(new, hq, d)
    n = len(pages)
    desc = B.PagedPrefillDesc.on_device(1, new, n, ints([0, new]), ints([0, n]), ints(pages), ints(np.full(n, 16)), ints([n - 3]), ints([48]))
    out, lse = torch.full_like(q, 7.0), torch.full((new, hq), 7.0, device=DEV)
    ws = torch.full((max(256, B.dag_prefill_paged_q8_workspace_bytes(desc, cache, new, hq)),), 0xff, dtype=torch.uint8, device=DEV)
    B.dag_attn_prefill_paged_q8(desc, q, cache, out, ws, lse=lse, softmax_scale=SCALE)
    return out.double().cpu().numpy(), lse.double().cpu().numpy(), 16 * n - new + 1 + np.arange(new)


def close(got, want, room):
    worst = float(np.max(np.abs(got - want) / room))
    assert worst <= 1.0, worst


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("new", [1, 40])
@pytest.mark.parametrize("none", [False, True])
def test_chunk_counts_the_keys_of_pages_of_zeros(new, d, none):
    """2^15 keys to a large one, 2^-11.5 of the sum.  The logarithm, 24, is rounded (2^-20), so are its two terms, the score is off by 2^-18 and
    the exponentials by a few 2^-24: 2^-16 has room."""
    cache = cache_of(d)
    pages = pages_of(1 << 20, ZEROS, TOP, 1 << 12)
    if none:  # a value that is no number, in one dim: the sums are taken once more
        cache.v_pool.view(torch.uint8)[ZEROS, 0, 7, 4] = 0x7f
    out, lse, seen = chunk(cache, pages, new, 4, d)
    tops, zeros = (np.array(x, dtype=np.float64) for x in zip(*(counts(pages, ZEROS, n) for n in seen)))
    total = tops * 2.0 ** FAR + zeros
    close(lse, np.log(total)[:, None], 2.0 ** -16)
    if none:
        assert np.isnan(out[:, :, 7]).all()
        out = np.delete(out, 7, axis=2)
    want = (1.5 * tops * 2.0 ** FAR / total)[:, None, None]
    close(out, want, want * (2.0 ** -8 + 2.0 ** -14))


def of_small(tops, tokens):
    return 256.0 * 2.0 ** -100 * tokens / (tops * 2.0 ** FAR + tokens)


# Probabilities and results are rounded to bf16, 2^-8 each (the probabilities are all equal: the same way), scores are off by 2^-18.
SMALL_ROOM = 2 * 2.0 ** -8 + 2.0 ** -15


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("new", [1, 7, 37, 40])  # (pages hidden from no row of a wave, or from some)
@pytest.mark.parametrize("none", [False, True])
def test_chunk_over_tiny_values(new, d, none):
    cache = cache_of(d)
    if none:
        cache.v_pool.view(torch.uint8)[SMALL, 0, 7, 4] = 0xff
    pages = pages_of(10, SMALL, TOP_OF_SMALL, 10)
    out, lse, seen = chunk(cache, pages, new, 4, d)
    if none:
        assert np.isnan(out[:, :, 7]).all()
        out = np.delete(out, 7, axis=2)
    want = np.array([of_small(*counts(pages, SMALL, n)) for n in seen])[:, None, None]
    close(out, want, want * SMALL_ROOM)


@pytest.mark.parametrize("scale", [0.0, 2.0 ** -149, 2.0 ** -127, 2.0 ** -126, 2.0 ** -61, 2.0 ** -60])
@pytest.mark.parametrize("new", [1, 40])
def test_chunk_over_value_scales_down_to_zero(new, scale):
    """Scores of zero: a page of 1.5, one of 256 times the scale, three full ones of the node's own of zeros.  The results are their mean."""
    cache = cache_of(64)
    cache.v_pool[TOP] = torch.full((1, 64, 16), 1.5, device=DEV).to(torch.float8_e4m3fn)
    cache.v_scale[SMALL] = scale
    q = torch.zeros((new, 4, 64), dtype=torch.bfloat16, device=DEV)
    pages = [TOP, SMALL, ZEROS, ZEROS, ZEROS]
    desc = B.PagedPrefillDesc.on_device(1, new, 5, ints([0, new]), ints([0, 5]), ints(pages), ints([16] * 5), ints([2]), ints([48]))
    out, lse = torch.full_like(q, 7.0), torch.full((new, 4), 7.0, device=DEV)
    ws = torch.full((max(256, B.dag_prefill_paged_q8_workspace_bytes(desc, cache, new, 4)),), 0xff, dtype=torch.uint8, device=DEV)
    B.dag_attn_prefill_paged_q8(desc, q, cache, out, ws, lse=lse)
    seen = (80 - new + 1 + np.arange(new))[:, None, None].astype(np.float64)
    want = (16 * 1.5 + 16 * 256 * scale) / seen
    close(out.double().cpu().numpy(), want, want * (2.0 ** -8 + 2.0 ** -20))
    close(lse.double().cpu().numpy(), np.log(seen[..., 0]), 2.0 ** -20)

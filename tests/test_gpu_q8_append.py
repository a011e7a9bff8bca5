"""GPU: dag_kv_append_rope_q8 against the oracle.

Values come from 16- or 32-bit inputs and a scale is a power of two, so x / scale is exact and a value's code is the nearest one: equal to
the oracle's.  A rotated key is off by its angles and products in 32 bits: cos and sin half a step (2^-25) each, two products
and a sum, at most 2.5 * 2^-24 (|lo| + |hi|) in all; a code is right if it is as near to the exact value as the oracle's up to twice that."""
import numpy as np
import pytest
import torch

from oracle import q8_oracle as q8
from paper_2602_07529_amd import binding as B
from tests.gpu_util import DEV

pytestmark = pytest.mark.gpu

PAGE = 16


def _bytes(t):
    return t.view(torch.uint8).cpu().numpy()


class Both:
    """A cache on the GPU and the oracle's."""

    def __init__(self, n_pages, hkv, d, seed=0, junk=True):
        self.cache = c = B.KvCacheQ8.empty(n_pages, hkv, d, DEV)
        rng = np.random.default_rng(seed)
        if junk:  # codes that are no number among them
            for t in (c.k_pool, c.v_pool):
                t.view(torch.uint8).copy_(torch.from_numpy(rng.integers(0, 256, size=tuple(t.shape), dtype=np.uint8)))
        self.read()

    def read(self):
        c = self.cache
        self.k, self.v = q8.tokens_of_pools(c.k_pool.float().cpu().numpy(), c.v_pool.float().cpu().numpy())
        self.ks, self.vs = c.k_scale.double().cpu().numpy(), c.v_scale.double().cpu().numpy()

    def append(self, slots, pos, k_new, v_new, theta):
        c = self.cache
        before = [_bytes(t).copy() for t in (c.k_pool, c.v_pool, c.k_scale, c.v_scale)]
        ints = lambda x: torch.tensor(np.asarray(x, dtype=np.int32), device=DEV)  # noqa: E731
        B.dag_kv_append_rope_q8(c, ints(slots), ints(pos), k_new.to(DEV), v_new.to(DEV), theta)
        turned = q8.rope(k_new.double().numpy(), np.asarray(pos), theta)
        half = turned.shape[-1] // 2
        size = np.abs(k_new.double().numpy())
        slack = np.concatenate([size[..., :half] + size[..., half:]] * 2, -1) * 2.5 * 2.0 ** -24
        at_k = q8.append(self.k, self.ks, turned, slots)
        at_v = q8.append(self.v, self.vs, v_new.double().numpy(), slots)
        want = self.k, self.v, self.ks, self.vs
        self.read()
        spread = np.zeros_like(self.k)
        for t, s in enumerate(slots):
            if 0 <= s < self.ks.shape[0] * PAGE:
                spread[s // PAGE, :, s % PAGE] = slack[t]
        for got, ref, scale, ref_scale, at, slack in ((self.k, want[0], self.ks, want[2], at_k, spread),
                                                      (self.v, want[1], self.vs, want[3], at_v, np.zeros_like(spread))):
            assert np.array_equal(scale, ref_scale)
            for page, _, exact in at:
                g, w = got[page] * scale[page][:, None, None], ref[page] * scale[page][:, None, None]
                assert np.array_equal(np.isnan(g), np.isnan(w))
                fine = ~np.isnan(w)
                assert (np.abs(g - exact) <= np.abs(w - exact) + 2 * slack[page])[fine].all()
                assert np.array_equal(g[fine & (slack[page] == 0)], w[fine & (slack[page] == 0)])
        untouched = np.ones(self.ks.shape[0], dtype=bool)
        untouched[[p for p, _, _ in at_k]] = False
        for a, t in zip(before, (c.k_pool, c.v_pool, c.k_scale, c.v_scale)):
            a, b = (x.reshape(len(untouched), -1)[untouched] for x in (a, _bytes(t)))
            assert np.array_equal(a, b)


def _new(seed, n, hkv, d, dtype, spread=0.0):
    gen = torch.Generator().manual_seed(seed)
    size = torch.exp(spread * torch.randn(n, 1, 1, generator=gen))
    return [(torch.randn(n, hkv, d, generator=gen) * size).to(dtype) for _ in range(2)]


@pytest.mark.parametrize("hkv,d,dtype", [(1, 64, torch.bfloat16), (2, 128, torch.bfloat16), (3, 64, torch.float32), (8, 128, torch.float32)])
def test_a_row_token_by_token_its_scale_growing(hkv, d, dtype):
    b = Both(5, hkv, d)
    n = 2 * PAGE + 3
    k, v = _new(1, n, hkv, d, dtype, spread=2.0)
    at = np.concatenate([p * PAGE + np.arange(PAGE) for p in (3, 0, 4)])
    for t in range(n):
        b.append([at[t]], [1000 + t], k[t:t + 1], v[t:t + 1], 5e5)


# lengths that begin, fill, end and continue pages, of many rows at once
@pytest.mark.parametrize("hkv,d,dtype", [(1, 128, torch.bfloat16), (4, 64, torch.bfloat16), (2, 128, torch.float32), (5, 64, torch.float32)])
@pytest.mark.parametrize("rows", [[(0, 1)], [(0, 16), (15, 1), (15, 2)], [(5, 3), (0, 40), (1, 15), (13, 100), (0, 15)], [(7, 9)] * 70,
                                  [(3, 1)] * 300])
def test_rows_of_any_length(hkv, d, dtype, rows):
    n_pages = sum(-(-(i0 + n) // PAGE) for i0, n in rows) + 2
    b = Both(n_pages, hkv, d, junk=False)
    perm = np.random.default_rng(7).permutation(n_pages)
    first, slots, pos, at = [], [], [], 0
    for i0, n in rows:
        count = -(-(i0 + n) // PAGE)
        place = (perm[at:at + count, None] * PAGE + np.arange(PAGE)).reshape(-1)
        first += list(place[:i0])
        slots += list(place[i0:i0 + n])
        pos += list(40000 - at + np.arange(n))
        at += count
    if first:
        k, v = _new(2, len(first), hkv, d, dtype)
        b.append(first, np.arange(len(first)), k, v, 1e4)
    k, v = _new(3, len(slots), hkv, d, dtype, spread=1.0)
    b.append(slots, pos, k, v, 1e4)


def test_slots_outside_the_pool_are_left_out_and_break_runs():
    b = Both(4, 2, 128)
    k, v = _new(4, 9, 2, 128, torch.bfloat16)
    b.append([16, -1, 4 * PAGE, 48, 49, 2 ** 31 - 1, -2 ** 31, 0, -5], np.arange(9), k, v, 1e4)
    before = [_bytes(t).copy() for t in (b.cache.k_pool, b.cache.v_pool, b.cache.k_scale)]
    b.append([-1] * 9, np.arange(9), k, v, 1e4)
    for x, t in zip(before, (b.cache.k_pool, b.cache.v_pool, b.cache.k_scale)):
        assert np.array_equal(x, _bytes(t))


def test_sizes_from_nothing_to_the_largest():
    hkv, d = 2, 64
    b = Both(12, hkv, d)
    k, v = _new(5, 12, hkv, d, torch.float32)
    size = [0.0, 1e-38, 1e-31, 2.0 ** -100, 1e-12, 1.0, 448.0, 449.0, 1e4, 1e20, 1e30, 3e37]
    for i, s in enumerate(size):
        k[i] *= s
        v[i] *= s
    v[6] = 448.0   # on the border: the scale is one
    v[7] = 448.0 * (1 + 2.0 ** -23)  # just above it
    b.append(np.arange(12) * PAGE, np.zeros(12), k, v, 1e4)
    assert b.vs[6, 0] == 1.0 and b.vs[7, 0] == 2.0 and b.vs[0, 0] == 2.0 ** -100
    # tokens of every size join those pages: old codes fall under the smallest normal, or stay as they are
    k2, v2 = _new(6, 12, hkv, d, torch.float32)
    b.append(np.arange(12) * PAGE + 1, np.zeros(12), k2 * 50, v2 * 50, 1e4)


def test_what_is_no_number_is_stored_as_that_and_leaves_the_scale():
    hkv, d = 2, 128
    b = Both(2, hkv, d)
    k, v = _new(8, 18, hkv, d, torch.bfloat16)
    v[3, 0, 5], v[4, 1, 6], v[16, 0, 0] = float("nan"), float("inf"), float("-inf")
    k[2, 1, 7] = float("nan")
    k[5, 0, :] = float("nan")
    b.append(np.arange(18), np.zeros(18), k, v, 1e4)  # (at position 0 a key is as it came: its partner takes nothing from it)
    assert np.isnan(b.v[0, 0, 3, 5]) and np.isnan(b.v[0, 1, 4, 6]) and np.isfinite(b.vs).all() and np.isfinite(b.ks).all()


def test_the_same_call_gives_the_same_bits_on_another_stream():
    hkv, d = 8, 128
    k, v = _new(9, 500, hkv, d, torch.bfloat16, spread=1.0)
    got = []
    for stream in (torch.cuda.current_stream(), torch.cuda.Stream()):
        with torch.cuda.stream(stream):
            b = Both(33, hkv, d, junk=False)
            b.append(np.arange(500) + 16, np.arange(500) * 7, k, v, 1e6)
            got.append([_bytes(t).copy() for t in (b.cache.k_pool, b.cache.v_pool, b.cache.k_scale, b.cache.v_scale)])
    for x, y in zip(*got):
        assert np.array_equal(x, y)

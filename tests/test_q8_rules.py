"""CPU: slices, work items and workspace of the 8-bit decode steps."""
import numpy as np
import pytest

from paper_2602_07529_amd import binding as B
from tests import q8_rules


def desc(groups, live, shared, own, size):
    return B.dag_decode_desc_t(groups, live, 16, shared, own, size)


@pytest.mark.parametrize("seed", range(400))
def test_slices_cover_the_longest_lists_and_the_workspace_holds_them(seed):
    rng = np.random.default_rng(seed)
    hkv = int(rng.choice([1, 2, 3, 4, 8, 16]))
    hq, d = hkv * int(rng.integers(1, 33)), int(rng.choice([64, 128]))
    groups, size = int(rng.integers(0, 20)), int(rng.choice([1, 2, 7, 40]))
    live = max(1, groups) * size
    shared, own = (int(2 ** rng.uniform(0, 12)) - 1 for _ in range(2))
    p = q8_rules.plan(desc(groups, live, shared, own, size), hq, hkv, d)
    assert p.rc == 0
    shared = shared if groups else 0
    for pages, chunk, splits in ((shared, p.chunk_a, p.splits_a), (own, p.chunk_b, p.splits_b)):
        assert chunk % 2 == 0 and 0 < chunk <= 258
        assert splits == -(-pages // chunk) and (pages == 0) == (splits == 0)
    assert p.rb_max * 32 >= size * (hq // hkv)
    assert p.items_a == groups * hkv * p.rb_max * p.splits_a and p.items_b == live * hkv * p.splits_b
    rows = live * hq * (p.splits_a + p.splits_b)
    assert p.off_ml % 256 == 0 and p.off_ml >= rows * d * 4 and p.bytes >= p.off_ml + rows * 8


@pytest.mark.parametrize("live,hkv,d,pages,whole", [
    (4, 8, 128, 41, True), (4, 8, 128, 42, False), (4, 8, 64, 52, True), (4, 8, 64, 53, False), (32, 8, 128, 101, True), (32, 8, 128, 102, False),
    (23, 8, 128, 42, False), (24, 8, 128, 42, True), (33, 8, 128, 10, False), (33, 8, 64, 41, True), (64, 8, 64, 41, True), (65, 8, 64, 1, False)])
def test_which_steps_take_one_launch(live, hkv, d, pages, whole):
    for shared in (0, pages // 2):
        assert bool(q8_rules.plan(desc(1 if shared else 0, live, shared, pages - shared, live), 4 * hkv, hkv, d).whole) is whole


@pytest.mark.parametrize("groups,live,pages", [(2 ** 20, 2 ** 24, 2 ** 20), (2 ** 30, 2 ** 30, 4000), (0, 2 ** 27, 1)])
def test_sizes_past_an_int_are_refused(groups, live, pages):
    assert q8_rules.plan(desc(groups, live, pages, pages, 16), 32, 8, 128).rc == -7

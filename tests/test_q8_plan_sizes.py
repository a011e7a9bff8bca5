"""CPU: 8-bit decode steps of any sizes are planned as exact arithmetic has it, or refused."""
import random

import pytest

from paper_2602_07529_amd import binding as B
from tests import q8_rules

MOST = 2 ** 31 - 1


def up(a, b):
    return -(-a // b)


def fits(groups, live, shared, own, size, hkv, g):
    rb = up(size * g, 32)
    a, b = groups * hkv * rb, live * hkv
    work = a * shared + b * own
    most = min(max(up(work, 1920 if rb > 1 and up(work, 1536) > 62 else 1536), 8), 256)

    def splits(pages):
        n = up(pages, most)
        return up(pages, 2 * up(up(pages, n), 2)) if n else 0

    sa, sb = splits(shared if a else 0), splits(own)
    return a * sa + b * sb <= MOST and live * (sa + sb) * hkv * g <= MOST and live * hkv * g <= MOST


@pytest.mark.parametrize("seed", range(20))
def test_what_does_not_fit_32_bits_is_refused_and_nothing_else(seed):
    rng = random.Random(seed)
    for i in range(2000):
        bits = 31 if i % 2 else 12
        groups, live, shared, own, size = (min(MOST, int(2 ** rng.uniform(0, bits)) - rng.randint(0, 1)) for _ in range(5))
        hkv, g, d = int(2 ** rng.uniform(0, 25 if i % 2 else 4)), rng.choice([1, 4, 32]), rng.choice([64, 128])
        shared = shared if groups else 0
        p = q8_rules.plan(B.dag_decode_desc_t(groups, live, 16, shared, own, size), hkv * g, hkv, d)
        assert p.rc == (0 if fits(groups, live, shared, own, size, hkv, g) else -7), (groups, live, shared, own, size, hkv, g)

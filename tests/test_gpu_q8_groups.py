"""GPU: cascades of many groups over an 8-bit cache in one launch, which finds a branch's group 64 groups at a time, with shared pages through the
caches and past them."""
import pytest
import torch

from tests import q8_rules
from tests.gpu_util import DEV
from tests.q8_cases import Cascade, check

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("groups", [63, 64, 65, 130])
@pytest.mark.parametrize("hq,hkv,d", [(4, 1, 128), (6, 2, 64), (8, 1, 64)])
def test_a_branch_finds_its_group_among_many(groups, hq, hkv, d):
    some = [(20 + g % 50, [] if g % 5 == 2 or g == 64 else [1 + g % 20] * (1 if g % 3 else 2 * (g < 20) + 1)) for g in range(groups)]
    c = Cascade(some, hq, hkv, d, groups)
    assert q8_rules.plan(c.desc.c, hq, hkv, d).whole
    c.call()
    torch.cuda.synchronize()
    check(c.out, c.q, c.contexts, c.cache)


@pytest.mark.parametrize("hq,hkv,d", [(4, 1, 128), (16, 2, 128), (4, 4, 64), (32, 8, 128), (12, 3, 64)])
@pytest.mark.parametrize("shared,own", [(300, 20), (20, 300), (64, 64), (500, 0)])
def test_shared_pages_through_the_caches_and_past_them(hq, hkv, d, shared, own):
    c = Cascade([(shared, [own, own // 2, 1]), (shared // 3, [own]), (0, [own, 3])], hq, hkv, d, shared)
    assert q8_rules.plan(c.desc.c, hq, hkv, d).whole
    c.call()
    torch.cuda.synchronize()
    check(c.out, c.q, c.contexts, c.cache)

"""dag_attn_prefill_paged_q8 against the oracle: chunks of new tokens over partly filled pages of an 8-bit cache."""
import numpy as np
import pytest
import torch

from paper_2602_07529_amd import binding as B
from tests.gpu_util import DEV
from tests.q8_chunk_cases import Chunks

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("hq,hkv,d", [(8, 2, 128), (4, 4, 64), (6, 2, 128), (5, 1, 64), (32, 1, 128), (7, 1, 128)])
@pytest.mark.parametrize("new", [1, 2, 9, 33, 70])
def test_lengths(hq, hkv, d, new):
    c = Chunks([([16] * 5 + [7], new + 3, new), ([16, 4, 16, 1], new, new), ([], new + 18, new)], hq, hkv, d, seed=new)
    c.call()
    c.check()


@pytest.mark.parametrize("d", [64, 128])
def test_ragged_nodes(d):
    rng = np.random.default_rng(d)
    nodes = [([int(x) for x in rng.integers(0, 17, size=rng.integers(0, 30))], int(n) + int(rng.integers(0, 40)), int(n))
             for n in rng.integers(0, 40, size=23)]
    c = Chunks(nodes, 8, 2, d, seed=3, idle=5, spare=9)
    c.call()
    c.check()


def test_single_tokens_of_many_nodes():
    rng = np.random.default_rng(5)
    nodes = [([16] * int(rng.integers(0, 12)) + [int(rng.integers(1, 17))], int(rng.integers(1, 40)), 1) for _ in range(150)]
    c = Chunks(nodes, 8, 2, 64, seed=4)
    c.call()
    c.check()


@pytest.mark.parametrize("new,pages", [(1, 700), (5, 701), (40, 259), (200, 130)])
def test_long_context_cut_among_workgroups(new, pages):
    c = Chunks([([16] * pages + [3], new, new)], 4, 1, 128, seed=new, q_scale=2.0)
    c.call()
    c.check(rows=sorted({0, new // 2, new - 1}))


def test_long_chunk():
    c = Chunks([([16] * 3 + [11], 700, 700), ([16] * 40, 300, 290)], 4, 2, 128, seed=1, idle=3)
    c.call()
    c.check(rows=[0, 1, 15, 16, 31, 32, 63, 64, 127, 128, 255, 256, 500, 698, 699, 700, 701, 850, 988, 989])


def test_rows_that_see_nothing():
    """Empty pages only, no pages at all, and new tokens whose own pages are empty too."""
    c = Chunks([([0, 0, 0], 5, 5), ([0], 16, 16), ([], 4, 4)], 4, 2, 64, seed=2)
    c.desc.t["ctx_page_len"].zero_()
    for row in c.contexts:
        row[:] = [(p, 0) for p, _ in row]
    c.call()
    c.check()
    assert (c.out[:c.n] == 0).all() and (c.lse[:c.n] == float("-inf")).all()


@pytest.mark.parametrize("scale", [0.3, -0.2, 0.0])
def test_softmax_scale(scale):
    c = Chunks([([16, 9], 20, 12)], 4, 2, 128, seed=6)
    c.call(softmax_scale=scale)
    c.check(scale)


def test_scale_that_is_no_number():
    c = Chunks([([16, 9], 20, 12), ([0], 3, 3)], 4, 2, 128, seed=6)
    c.desc.t["ctx_page_len"][-2] = 0  # (the second node's own page)
    c.call(softmax_scale=float("nan"))
    assert c.out[:12].isnan().all() and c.lse[:12].isnan().all()
    assert (c.out[12:15] == 0).all() and (c.lse[12:15] == float("-inf")).all()


@pytest.mark.parametrize("d", [64, 128])
def test_no_number_reaches_only_the_rows_that_see_it(d):
    c = Chunks([([16] * 5, 40, 30)], 4, 2, d, seed=8)
    page = int(c.lists[0][6])  # own tokens 16 .. 31, the new ones 6 .. 21
    c.cache.v_pool.view(torch.uint8)[page, 1, 5, 4] = 0x7f  # own token 20, dim 5
    c.cache.k_pool.view(torch.uint8)[page, 0, 0, 9, 3] = 0xff  # own token 25
    c.call()
    got = c.out[:30].float()
    seen_v, seen_k = torch.arange(30, device=DEV) + 10 >= 20, torch.arange(30, device=DEV) + 10 >= 25
    assert (got[:, 2:, 5].isnan() == seen_v[:, None]).all()
    rest = got.clone()
    rest[:, 2:, 5] = 0
    assert not rest[:, 2:].isnan().any()
    assert (got[:, :2].isnan() == seen_k[:, None, None]).all()
    c.check(rows=range(10))


def test_scales_far_apart():
    c = Chunks([([16] * 9 + [2], 33, 20)], 4, 1, 128, seed=9)
    c.cache.k_scale[c.lists[0][0]] = 2.0 ** -100
    c.cache.v_scale[c.lists[0][1]] = 2.0 ** -100
    c.cache.v_scale[c.lists[0][2]] = 2.0 ** 20
    c.call()
    c.check()


def test_scores_that_grow_along_the_context():
    """Every stretch of the context has larger scores than all before it, by more than 2^100 from end to end."""
    c = Chunks([([16] * 64, 20, 20)], 4, 1, 128, seed=10)
    c.cache.k_scale[torch.as_tensor(c.lists[0].astype(np.int64), device=DEV)] = torch.exp2(torch.linspace(-9, -2, 66, device=DEV))[:, None]
    c.call()
    c.check()


def test_no_lse_and_the_same_bits_again():
    c = Chunks([([16] * 300, 100, 90), ([16] * 20, 3, 3)], 8, 2, 128, seed=11)
    c.call()
    first = c.out.clone()
    c.out.fill_(7.0)
    c.ws.fill_(0x55)
    c.call(lse=None)
    assert torch.equal(first, c.out)


def test_page_ids_outside_the_pool_are_not_followed():
    c = Chunks([([16] * 6, 16, 16)], 4, 2, 64, seed=12)
    pages = c.desc.t["ctx_pages"]
    pages[1], pages[3] = 2 ** 31 - 1, -5
    last = c.cache.c.n_pages - 1
    for row in c.contexts:
        row[1], row[3] = ([last], row[1][1]), ([0], row[3][1])
    for x in (c.cache.k_pool, c.cache.v_pool):
        x[last], x[0] = x[int(c.lists[0][0])], x[int(c.lists[0][2])]
    for x in (c.cache.k_scale, c.cache.v_scale):
        x[last], x[0] = x[int(c.lists[0][0])], x[int(c.lists[0][2])]
    c.call()
    c.check()

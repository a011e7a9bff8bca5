"""dag_attn_prefill_paged_q8: queries of all sizes, calls that overlap, captured calls whose lengths change, long pools, random batches."""
import numpy as np
import pytest
import torch

from oracle import q8_oracle as q8
from paper_2602_07529_amd import binding as B
from tests.gpu_util import DEV
from tests.q8_cases import values
from tests.q8_chunk_cases import Chunks

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("new", [3, 50])
@pytest.mark.parametrize("size", [2.0 ** -110, 2.0 ** -60, 2.0 ** 5, 2.0 ** 30])
def test_sizes_of_queries(new, size):
    """With the softmax scale that brings the scores back: the parts of a query in 8 bits have its size."""
    c = Chunks([([16] * 4 + [5], new, new), ([], new + 3, new)], 8, 2, 128, seed=21, q_scale=size)
    scale = 128 ** -0.5 / size
    c.call(softmax_scale=scale)
    c.check(scale)


@pytest.mark.parametrize("new", [3, 50])
def test_elements_of_a_query_far_apart(new):
    """One element of every row is 2^16 times the others: these lose nothing but what is below 2^-22 of the largest, d / 2 times."""
    c = Chunks([([16] * 4 + [5], new, new)], 4, 1, 128, seed=22)
    c.q[:, :, 77] *= 2.0 ** 16
    c.cache.k_pool.view(torch.uint8)[:, :, 4, :, 13] = 0  # (dim 77: its keys are 0, so the others decide)
    c.call()
    d, (k, v) = 128, values(c.cache)
    keys = np.nan_to_num(np.abs(k), nan=0.0)  # (slots without a token hold codes that are no number)
    err = 2.0 ** -22 * float(c.q.abs().max()) * keys.sum(-1).max() * d ** -0.5  # of a score: a probability is off by a factor of e^err, so is the sum
    ref, mass, _ = q8.attention(c.q.double().cpu().numpy(), c.contexts, k, v, d ** -0.5)
    room = mass * (np.expm1(2 * err) + 2.0 ** -7 * np.exp(2 * err)) + 2.0 ** -8 * np.abs(ref)
    assert (np.abs(c.out.double().cpu().numpy() - ref) <= room).all()


@pytest.mark.parametrize("new", [2, 40])
def test_rows_that_are_no_number(new):
    c = Chunks([([16, 9], new, new), ([0], 3, 1)], 4, 2, 64, seed=23)
    c.desc.t["ctx_page_len"][-2] = 0
    c.contexts[-1] = [(p, 0) for p, _ in c.contexts[-1]]
    c.q[1, 2, 5], c.q[0, 1, 3], c.q[-1, 0, 0] = float("nan"), float("inf"), float("nan")
    c.call()
    got = c.out.float()
    assert got[1, 2].isnan().all() and got[0, 1].isnan().all()
    assert (got[-1] == 0).all() and (c.lse[-1] == float("-inf")).all()
    got[1, 2], got[0, 1] = 0, 0
    assert not got.isnan().any()


def test_values_that_are_no_number_behind_a_long_context():
    """In stretches of their own, in every wave's part, seen and hidden."""
    c = Chunks([([16] * 300, 30, 20)], 4, 1, 128, seed=24)
    v = c.cache.v_pool.view(torch.uint8)
    v[int(c.lists[0][301]), 0, 9, 9] = 0x7f  # own token 25: the new ones are 10 .. 29
    c.call()
    seen = torch.arange(20, device=DEV) + 10 >= 25
    assert (c.out[:20, :, 9].isnan() == seen[:, None]).all()
    c.out[:, :, 9] = 0
    assert not c.out.isnan().any()
    v[int(c.lists[0][150]), 0, 3, 2] = 0xff
    c.call()
    assert c.out[:20, :, 3].isnan().all()


def test_captured_call_with_other_lengths():
    """A captured call reads its lengths, pages and offsets anew at every replay, within the bounds of the capture."""
    c = Chunks([([16] * 9, 40, 33), ([16] * 40, 20, 9)], 8, 2, 128, seed=25, idle=2)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        c.call()
    for step in range(4):
        c.out.fill_(7.0)
        c.lse.fill_(7.0)
        graph.replay()
        torch.cuda.synchronize()
        if step == 0:
            c.check()
            first = c.out.clone()
        elif step == 1:
            assert torch.equal(c.out, first)
        keep = [list(r) for r in c.contexts]
        if step == 1:  # the second page of the first node's front loses its tokens, the second node three rows
            c.desc.t["ctx_page_len"][1] = 0
            for r in c.contexts[:33]:
                r[1] = (r[1][0], 0)
        if step == 2:
            c.check()
            c.desc.t["q_off"][2] = 33 + 6
            c.desc.t["own_len"][1] = 17
            c.contexts = keep[:33] + [row[:40] + [(row[40][0], min(16, 12 + i)), (row[41][0], max(0, 12 + i - 16))] for i, row in enumerate(keep[33:39])]
            c.desc.t["ctx_page_len"][-2] = 1  # (of the second node's last page; the entry behind it is the arrays' spare one)
            c.n = 39
        if step == 3:
            c.check()


def test_calls_at_once():
    """Two streams, a workspace each."""
    cs = [Chunks([([16] * 500, 5, 5), ([16] * 20, 90, 80)], 8, 2, 128, seed=s) for s in (26, 27)]
    alone = []
    for c in cs:
        c.call()
        alone.append(c.out.clone())
        c.out.fill_(7.0)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in cs]
    for _ in range(5):
        for c, s in zip(cs, streams):
            with torch.cuda.stream(s):
                c.call()
    torch.cuda.synchronize()
    for c, want in zip(cs, alone):
        assert torch.equal(c.out, want)


def test_pool_of_more_than_4_gib():
    hkv, d, n_pages = 8, 128, 140000  # 4.3 GiB a pool
    cache = B.KvCacheQ8.empty(n_pages, hkv, d, DEV)
    small = Chunks([([16] * 5, 40, 20)], 8, hkv, d, seed=28)
    far = torch.arange(n_pages - small.cache.c.n_pages, n_pages, device=DEV)
    for name in ("k_pool", "v_pool"):
        getattr(cache, name).view(torch.uint8)[far] = getattr(small.cache, name).view(torch.uint8)
    for name in ("k_scale", "v_scale"):
        getattr(cache, name)[far] = getattr(small.cache, name)
    small.call()
    want = small.out.clone()
    small.desc.t["ctx_pages"].add_(int(far[0]))
    small.cache = cache
    small.call()
    assert torch.equal(small.out, want)


@pytest.mark.parametrize("seed", range(12))
def test_random_batches(seed):
    rng = np.random.default_rng(100 + seed)
    hkv, g, d = int(rng.choice([1, 2, 3])), int(rng.choice([1, 2, 4, 5, 8])), int(rng.choice([64, 128]))
    nodes = []
    for _ in range(int(rng.integers(1, 12))):
        new = int(rng.choice([1, 2, 7, 17, 60, 150]))
        front = [16 if rng.random() < 0.8 else int(rng.integers(0, 17)) for _ in range(int(rng.choice([0, 3, 30, 90])))]
        nodes.append((front, new + int(rng.choice([0, 1, 15, 16, 40])), new))
    c = Chunks(nodes, hkv * g, hkv, d, seed=seed, idle=int(rng.integers(0, 4)), spare=int(rng.choice([0, 100])), scales=str(rng.choice(["free", "powers"])))
    c.call()
    rows = rng.permutation(c.n)[:60]
    c.check(rows=sorted(int(r) for r in rows))
    assert c.out[:c.n].isfinite().all()

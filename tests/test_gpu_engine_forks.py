"""The calls together: branches over an 8-bit cache that take headers at once, tokens one by one, are selected, copied and moved; plans whose
longer texts go through the tiled call."""
import numpy as np
import pytest
import torch

from oracle import dag_oracle as orc
from oracle import q8_oracle as q8
from paper_2602_07529_amd import binding as B
from paper_2602_07529_amd import engine
from tests.gpu_util import DEV
from tests.q8_cases import check, values

pytestmark = pytest.mark.gpu


def rows_of(shape, gen):
    return torch.randn(shape, device=DEV, generator=gen).to(torch.bfloat16)


@pytest.mark.parametrize("capture", [False, True])
@pytest.mark.parametrize("rotary", [False, True])
def test_branches(capture, rotary):
    n, hq, hkv, d, prefix, most = 5, 8, 2, 64, 39, 60
    gen = torch.Generator(device=DEV).manual_seed(3)
    cache = B.KvCacheQ8.empty(60, hkv, d, DEV)
    rope = B.Rope(32, 10000.0, DEV, layout=B.ROPE_PAIRS, stretch=4.0, original=64.0, factor=1.1) if rotary else None
    k0, v0 = rows_of((prefix, hkv, d), gen), rows_of((prefix, hkv, d), gen)
    f = engine.Fork(cache, k0, v0, n, most, hq, rope or 10000.0, capture=capture)
    freq = q8.frequencies(32, 10000.0, 4.0, 64.0)

    def turned(k, first):
        k, pos = k.double().cpu().numpy(), first + np.arange(len(k))
        return q8.rotary(k, pos, freq, True, 1.1) if rotary else orc.rope(k, pos, 10000.0)

    history = [[turned(k0, 0), v0.double().cpu().numpy()] for _ in range(n)]  # what every branch has seen

    def remember(b, k, v):
        history[b] = [np.concatenate([history[b][0], turned(k, len(history[b][0]))]), np.concatenate([history[b][1], v.double().cpu().numpy()])]

    def contexts():
        table, length = f.rows.table.cpu().numpy(), f.len.cpu().numpy()
        return [[(table[0, :3], prefix), (table[1 + b, :-(-int(length[1 + b]) // 16)], int(length[1 + b]))] for b in range(n)]

    def held():
        """The cache holds every branch's history: a code is off by half a step of 2^-3 of its value, or of 2^-9 of the page's scale, twice where
        the scale has grown since."""
        k, v = values(cache)
        for b, c in enumerate(contexts()):
            for x, want in ((k, history[b][0]), (v, history[b][1])):
                got = np.concatenate([x[p].transpose(0, 2, 1, 3).reshape(-1, hkv, d)[:m] for p, m in c])
                top = np.abs(want).max()
                assert got.shape == want.shape and (np.abs(got - want) <= np.abs(want) * 2.0 ** -3 + top * 2.0 ** -8).all()

    def steps(count):
        for _ in range(count):
            q, k, v = rows_of((n, hq, d), gen), rows_of((n, hkv, d), gen), rows_of((n, hkv, d), gen)
            out = f.step(q, k, v)
            for b in range(n):
                remember(b, k[b:b + 1], v[b:b + 1])
            check(out, q, contexts(), cache)

    def header(m):
        q, k, v = rows_of((n, m, hq, d), gen), rows_of((n, m, hkv, d), gen), rows_of((n, m, hkv, d), gen)
        out = f.extend(q, k, v)
        for b in range(n):
            remember(b, k[b], v[b])
        seen = []
        for b, c in enumerate(contexts()):
            seen += [[c[0], (c[1][0], c[1][1] - m + 1 + i)] for i in range(m)]
        check(out.reshape(n * m, hq, d), q.reshape(n * m, hq, d), seen, cache)

    def select(parents):
        f.select(parents)
        before = list(history)
        for b, p in enumerate(parents):
            history[b] = before[p]
        assert int(f.refused) == 0

    steps(3)
    header(20)
    held()
    select([0, 0, 2, 0, 2])
    held()
    steps(2)
    select([0, 1, 1, 1, 4])
    page_map = f.compact().cpu().numpy()
    used = cache.c.n_pages - int(f.free)
    assert sorted(page_map[page_map >= 0]) == list(range(used)) and int(f.rows.table[0, 0]) < used
    held()
    header(7)
    steps(4)
    held()
    assert not f.rows.table[:, 0].lt(0).any()
    with pytest.raises(ValueError):
        f.select([1, 0, 2, 3, 4])
    with pytest.raises(ValueError):
        f.extend(*(rows_of((n, most, h, d), gen) for h in (hq, hkv, hkv)))
    f.select(list(range(n)))


@pytest.mark.parametrize("d,hq,hkv", [(64, 4, 1), (128, 8, 2)])
def test_plan_with_tiled_steps(d, hq, hkv):
    """Prompt and headers of a plan with a join in pieces: every token's output is the DAG-masked attention over what the cache holds."""
    parents = [[], [0], [0], [1], [1, 2]]
    length = np.asarray([70, 45, 33, 5, 40], dtype=np.int32)
    T = int(length.sum())
    gen = torch.Generator(device=DEV).manual_seed(d)
    q, k, v = rows_of((T, hq, d), gen), rows_of((T, hkv, d), gen), rows_of((T, hkv, d), gen)
    results = []
    for tiled in (None, 1, 16):
        cache = B.KvCacheQ8.empty(24, hkv, d, DEV)
        out, n_steps, _, _ = engine.run_plan(parents, length, q, k, v, 1e4, chunk=[32, 20, 1, 3, 40], cache=cache, tiled=tiled)
        results.append((out.double().cpu().numpy(), cache))
    assert torch.equal(results[0][1].k_pool.view(torch.uint8), results[1][1].k_pool.view(torch.uint8))
    plain = results[0][0]
    for got, _ in results[1:]:  # two roundings of the output and two of the probabilities between them
        assert np.abs(got - plain).max() <= 4 * 2.0 ** -8 * np.abs(plain).max()
        assert np.linalg.norm(got - plain) <= 2.0 ** -7 * np.linalg.norm(plain)

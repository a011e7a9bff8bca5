"""GPU: tables, append and attention over the 8-bit cache as they are used together: branches behind a shared prefix step by step
(also captured and replayed), rows that end and begin, whole plans through the scheduler."""
import numpy as np
import pytest
import torch

from oracle import dag_oracle as orc
from oracle import q8_oracle as q8
from paper_2602_07529_amd import binding as B
from paper_2602_07529_amd import engine
from workloads import dags
from tests.gpu_util import DEV
from tests.q8_cases import check, ints, pages_of

pytestmark = pytest.mark.gpu

PAGE = 16


def _randn(gen, *shape):
    return torch.randn(*shape, generator=gen).to(torch.bfloat16).to(DEV)


@pytest.mark.parametrize("n,prefix,steps,hq,hkv,d", [(3, 37, 20, 8, 2, 128), (1, 0, 18, 4, 4, 64), (9, 700, 5, 40, 8, 128), (5, 16, 33, 5, 1, 64)])
def test_branches_behind_a_prefix_step_by_step_and_replayed(n, prefix, steps, hq, hkv, d):
    gen = torch.Generator().manual_seed(n)
    k, v = _randn(gen, prefix, hkv, d), _randn(gen, prefix, hkv, d)
    toks = [(_randn(gen, n, hq, d), _randn(gen, n, hkv, d), _randn(gen, n, hkv, d)) for _ in range(steps)]
    n_pages = pages_of(prefix) + n * pages_of(steps) + 1
    forks = [engine.Fork(B.KvCacheQ8.empty(n_pages, hkv, d, DEV), k, v, n, steps, hq, 1e4, capture=c) for c in (False, True)]
    for i, tok in enumerate(toks):
        outs = [f.step(*tok).clone() for f in forks]
        torch.cuda.synchronize()
        assert torch.equal(*outs)
        f = forks[0]
        assert f.refused.item() == 0 and f.len.tolist() == [prefix] + [i + 1] * n and f.pos.tolist() == [prefix + i] * n
        table = f.rows.table.cpu().numpy()
        contexts = [[(table[0, :pages_of(prefix)], prefix), (table[1 + b, :pages_of(i + 1)], i + 1)] for b in range(n)]
        held = np.concatenate([p for p, _ in contexts[0][:1]] + [c[1][0] for c in contexts])
        assert len(set(held.tolist())) == len(held)
        if i in (0, 1, 15, 16, steps - 1):
            check(outs[0], tok[0], contexts, f.cache)
    a, b = (f.cache for f in forks)
    assert torch.equal(a.k_pool.view(torch.uint8), b.k_pool.view(torch.uint8)) and torch.equal(a.v_scale, b.v_scale)
    with pytest.raises(ValueError):
        forks[0].step(*toks[0])


def test_the_cache_holds_what_was_appended():
    """Every value comes back within e4m3's half step of its page's scale (half as much again where a code was rounded twice)."""
    gen = torch.Generator().manual_seed(3)
    n, hkv, d, steps = 4, 2, 128, 40
    toks = [[(torch.randn(n, h, d, generator=gen) * s).to(torch.bfloat16) for h in (8, hkv, hkv)] for s in torch.exp(torch.randn(steps, generator=gen))]
    f = engine.Fork(B.KvCacheQ8.empty(20, hkv, d, DEV), torch.zeros(0, hkv, d, dtype=torch.bfloat16, device=DEV),
                    torch.zeros(0, hkv, d, dtype=torch.bfloat16, device=DEV), n, steps, 8, 1e4, capture=True)
    for tok in toks:
        f.step(*(x.to(DEV) for x in tok))
    torch.cuda.synchronize()
    k, v = q8.tokens_of_pools(f.cache.k_pool.float().cpu().numpy(), f.cache.v_pool.float().cpu().numpy())
    ks, vs = f.cache.k_scale.cpu().numpy(), f.cache.v_scale.cpu().numpy()
    table = f.rows.table.cpu().numpy()
    for b in range(n):
        for i, (_, kt, vt) in enumerate(toks):
            page, slot = table[1 + b, i // PAGE], i % PAGE
            for got, scale, x in ((k, ks, q8.rope(kt[b:b + 1].double().numpy(), [i], 1e4)[0]), (v, vs, vt[b].double().numpy())):
                room = np.maximum(np.abs(x) * 2.0 ** -4, 1.5 * 2.0 ** -10 * scale[page][:, None]) * (1 + 2.0 ** -20)
                assert (np.abs(got[page, :, slot] * scale[page][:, None] - x) <= room).all()


def test_rows_end_and_begin_while_others_go_on():
    gen = torch.Generator().manual_seed(5)
    rng = np.random.default_rng(5)
    n, hq, hkv, d, n_pages, width = 6, 8, 2, 64, 40, 9
    cache = B.KvCacheQ8.empty(n_pages, hkv, d, DEV)
    rows = B.KvRows(torch.zeros((n, width), dtype=torch.int32, device=DEV), torch.arange(n_pages, dtype=torch.int32, device=DEV))
    length, free = ints([0] * n), ints([n_pages])
    for step in range(12):
        new = [int(rng.integers(0, 30)) if step % 3 == 0 else 1 for _ in range(n)]
        if step % 3 == 2:
            B.dag_kv_release(rows, ints(rng.integers(0, 2, n)), length, length, free, free)
        total = sum(new)
        off, slots, pos, page_off, pages, refused = (ints([0] * m) for m in (n + 1, total, total, n + 1, n_pages, 1))
        B.dag_kv_tables(rows, ints(new), length, length, free, free, off, slots, pos=pos, page_off=page_off, pages=pages, refused=refused)
        k, v, q = _randn(gen, total, hkv, d), _randn(gen, total, hkv, d), _randn(gen, n, hq, d)
        B.dag_kv_append_rope_q8(cache, slots, pos, k, v, 1e4)
        # a segment to a row, which its last token reads
        lens = length.tolist()
        seg = B.SegDecodeDesc.on_device(n, n, width, 1, n, page_off, pages, length, ints(range(n + 1)), ints(range(n)), ints(range(n + 1)), ints(range(n)))
        own = B.DecodeDesc.on_device(0, n, 0, width, 0, branch_page_off=page_off, branch_pages=pages, branch_len=length)
        outs = []
        for call, need, desc in ((B.dag_attn_decode_segments_q8, B.dag_decode_segments_q8_workspace_bytes, seg),
                                 (B.dag_attn_decode_q8, B.dag_decode_q8_workspace_bytes, own)):
            out = torch.full_like(q, float("nan"))
            call(desc, q, cache, out, torch.empty(max(256, need(desc, cache, hq)), dtype=torch.uint8, device=DEV))
            outs.append(out)
        po, pg = page_off.tolist(), pages.cpu().numpy()
        held = pg[:po[-1]]
        assert len(set(held.tolist())) == len(held) and free.item() + len(held) == n_pages
        contexts = [[(pg[po[r]:po[r + 1]], lens[r])] for r in range(n)]
        for out in outs:
            check(out, q, contexts, cache)


def test_a_plan_through_the_scheduler():
    parents = [[], [0], [0], [1], [1], [2], [2], [2], [3, 4, 5]]
    L = np.asarray([37, 16, 5, 21, 1, 33, 18, 7, 12], dtype=np.int32)
    hq, hkv, d, theta = 8, 2, 128, 1e4
    T = int(L.sum())
    q, k, v = dags.make_qkv(11, T, hq, hkv, d, 0.7, torch.bfloat16)
    # one element of every key and value is 4 (of keys one that hardly turns): no page's scale grows, every code is rounded once
    k[..., d // 2 - 1], v[..., 0] = 4.0, 4.0
    cache = B.KvCacheQ8.empty(60, hkv, d, DEV)
    first = {}

    def on_step(st):
        for i in range(st["n_segments"]):
            a, b = st["seg_page_off"][i:i + 2]
            first[int(st["seg_node"][i])] = st["seg_pages"][a:b].copy()

    out, n_steps, _, _ = engine.run_plan(parents, L, q.to(DEV), k.to(DEV), v.to(DEV), theta, chunk=[16, 4, 4, 1, 1, 1, 1, 1, 5], on_step=on_step,
                                         cache=cache)
    assert n_steps == len(orc.schedule_steps(parents, L, [16, 4, 4, 1, 1, 1, 1, 1, 5]))
    anc = dags.closure_from_parents(parents)
    contexts = [[(first[u], int(L[u])) for u in sorted(anc[v_])] + [(first[v_], i + 1)] for v_ in range(len(L)) for i in range(L[v_])]
    check(out, q.to(DEV), contexts, cache)

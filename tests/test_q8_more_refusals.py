"""CPU: what the entry points for chunks over the 8-bit cache, for rotary positions and for shared pages refuse, before any GPU work."""
import ctypes as C

import numpy as np
import pytest
import torch

from oracle import q8_oracle as q8
from paper_2602_07529_amd import binding as B
from paper_2602_07529_amd import engine
from tests.test_q8_refusals import FAKE, kv


def replaced(args, i, x):
    return tuple(x if j == i else y for j, y in enumerate(args))


def chunk(nodes=3, page=16, new=40, pages=900, arrays=FAKE, **other):
    d = B.dag_paged_prefill_desc_t(nodes, page, new, pages, *([arrays] * 6))
    for name, x in other.items():
        setattr(d, name, x)
    return C.byref(d)


def test_chunk():
    need_of, f = B.lib().dag_prefill_paged_q8_workspace_bytes, B.lib().dag_attn_prefill_paged_q8
    need = need_of(chunk(), 100, 8, 2, 128)
    assert need > 0
    ok = (FAKE, 100, FAKE, 0, 8, 0.1, FAKE, need, None)
    assert f(None, kv(), *ok) == -1 and f(chunk(), None, *ok) == -1
    for i in (0, 2):
        assert f(chunk(), kv(), *replaced(ok, i, 0)) == -1 and f(chunk(), kv(), *replaced(ok, i, FAKE + 8)) == -8
    assert f(chunk(), kv(), *replaced(ok, 3, FAKE + 2)) == -8
    for name in ("q_off", "ctx_page_off", "ctx_pages", "ctx_page_len", "own_page", "own_len"):
        assert f(chunk(**{name: 0}), kv(), *ok) == -1
    for name in ("k_pool", "v_pool", "k_scale", "v_scale"):
        assert f(chunk(), kv(**{name: 0}), *ok) == -1 and f(chunk(), kv(**{name: FAKE + 2}), *ok) == -8
    assert f(chunk(), kv(), *replaced(ok, 7, need - 1)) == -6 and f(chunk(), kv(), *replaced(ok, 6, 0)) == -6
    assert f(chunk(), kv(), *replaced(ok, 6, FAKE + 8)) == -8
    for hq in (7, 0, -8, 2 * 257):
        assert f(chunk(), kv(), *replaced(ok, 4, hq)) == -7 and need_of(chunk(), 100, hq, 2, 128) == 0
    assert f(chunk(), kv(d=96), *ok) == -7 and f(chunk(), kv(hkv=0), *ok) == -7 and need_of(chunk(), 100, 8, 2, 96) == 0
    assert f(chunk(page=32), kv(), *ok) == -7 and need_of(chunk(page=32), 100, 8, 2, 128) == 0
    for bad in (dict(nodes=-1), dict(new=-1), dict(pages=-1)):
        assert f(chunk(**bad), kv(), *ok) == -2 and need_of(chunk(**bad), 100, 8, 2, 128) == 0
    assert f(chunk(), kv(pages=0), *ok) == -2 and f(chunk(), kv(pages=-1), *ok) == -2 and f(chunk(), kv(), *replaced(ok, 1, -1)) == -2
    for empty in (dict(nodes=0), dict(new=0)):
        assert f(chunk(arrays=0, **empty), kv(k_pool=0), 0, 100, 0, 0, 8, 0.1, 0, 0, None) == 0
    assert f(chunk(arrays=0), kv(k_pool=0), 0, 0, 0, 0, 8, 0.1, 0, 0, None) == 0  # no rows


@pytest.mark.parametrize("nodes,new,pages,rows,hq,hkv", [
    (2 ** 31 - 1, 1, 10, 100, 8, 8), (4, 2 ** 31 - 1, 10, 2 ** 31 - 1, 8, 8), (4, 100, 2 ** 31 - 1, 100, 8, 8), (4, 9, 10, 2 ** 31, 8, 8),
    (4, 9, 10, 100, 2 ** 30, 2 ** 30), (2 ** 22, 1, 10, 2 ** 22, 8, 8), (4, 2 ** 28, 10, 2 ** 30, 256, 1)])
def test_chunk_sizes_past_a_launch(nodes, new, pages, rows, hq, hkv):
    assert B.lib().dag_prefill_paged_q8_workspace_bytes(chunk(nodes=nodes, new=new, pages=pages), rows, hq, hkv, 64) == 0
    assert B.lib().dag_attn_prefill_paged_q8(chunk(nodes=nodes, new=new, pages=pages), kv(hkv=hkv, d=64), FAKE, rows, FAKE, 0, hq, 0.1, FAKE, 2 ** 62,
                                             None) == -7


def test_chunk_workspaces_stay_small():
    """Contexts are cut only where there are few pairs, so partial results take no more than a few workgroups' worth of them a compute unit."""
    rng = np.random.default_rng(1)
    for _ in range(500):
        nodes, new, pages = (int(2 ** rng.uniform(0, hi)) for hi in (9, 13, 13))
        rows, hkv, g = int(rng.integers(1, nodes * new + 1)), int(rng.integers(1, 9)), int(rng.integers(1, 9))
        need = B.lib().dag_prefill_paged_q8_workspace_bytes(chunk(nodes=nodes, new=new, pages=pages), rows, hkv * g, hkv, 128)
        assert need <= 1 << 30


def rope(rotary=64, layout=0, freq=FAKE):
    return C.byref(B.dag_rope_t(freq, 1.0, rotary, layout))


def test_rope_apply():
    f = B.lib().dag_rope_apply
    ok = (FAKE, 5, FAKE, 1024, FAKE, 1024, FAKE, 256, FAKE, 256, 8, 2, 128, 0, B.DAG_BF16, None)
    assert f(None, *ok) == -1
    for i in (0, 4, 8):
        assert f(rope(), *replaced(ok, i, 0)) == -1
    assert f(rope(freq=0), *ok) == -1 and f(rope(freq=FAKE + 4), *ok) == -8
    for i in (2, 4, 6, 8):
        assert f(rope(), *replaced(ok, i, FAKE + 8)) == -8
    for i, least in ((3, 1024), (5, 1024), (7, 256), (9, 256)):
        assert f(rope(), *replaced(ok, i, least - 8)) == -2 and f(rope(), *replaced(ok, i, least + 4)) == -8
    for n in (-1, 2 ** 31):
        assert f(rope(), *replaced(ok, 1, n)) == -2
    for rotary in (0, 8, 24, 144, -16):
        assert f(rope(rotary), *ok) == -7
    assert f(rope(layout=2), *ok) == -7 and f(rope(), *replaced(ok, 12, 120)) == -7 and f(rope(), *replaced(ok, 12, 272)) == -7
    assert f(rope(), *replaced(ok, 14, 3)) == -7 and f(rope(), *replaced(ok, 10, 0)) == -7 and f(rope(), *replaced(ok, 11, 0)) == -7
    assert f(rope(freq=0), 0, 0, *ok[2:]) == 0 and f(rope(), 0, 5, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 128, 0, B.DAG_BF16, None) == 0


def test_append_rotary():
    f = B.lib().dag_kv_append_rotary_q8

    def call(cache=None, r=None, slots=FAKE, pos=FAKE, n=5, k=FAKE, ks=256, v=FAKE, vs=256, dtype=B.DAG_BF16):
        return f(cache or kv(), slots, pos, n, k, ks, v, vs, r or rope(), dtype, None)

    assert f(None, FAKE, FAKE, 5, FAKE, 256, FAKE, 256, rope(), B.DAG_BF16, None) == -1
    assert f(kv(), FAKE, FAKE, 5, FAKE, 256, FAKE, 256, None, B.DAG_BF16, None) == -1
    for name in ("slots", "pos", "k", "v"):
        assert call(**{name: 0}) == -1
    for name in ("k", "v"):
        assert call(**{name: FAKE + 8}) == -8 and call(**{name + "s": 248}) == -2 and call(**{name + "s": 260}) == -8
    for name in ("k_pool", "v_pool", "k_scale", "v_scale"):
        assert call(kv(**{name: 0})) == -1 and call(kv(**{name: FAKE + 2})) == -8
    for r in (0, 16, 48, 160):
        assert call(r=rope(r)) == -7
    assert call(kv(d=64), rope(128), ks=128, vs=128) == -7 and call(r=rope(layout=-1)) == -7 and call(kv(d=80)) == -7 and call(dtype=5) == -7
    assert call(r=rope(freq=0)) == -1 and call(r=rope(freq=FAKE + 4)) == -8 and call(n=-1) == -2 and call(n=2 ** 31) == -2 and call(kv(pages=-1)) == -2
    assert call(kv(k_pool=0), rope(freq=0), slots=0, pos=0, n=0, k=0, v=0) == 0


@pytest.mark.parametrize("kind", [dict(theta=1e4), dict(theta=5e5, stretch=8.0), dict(theta=1e6, stretch=32.0, original=8192.0, low=1.0, high=4.0)])
def test_frequencies(kind):
    args = dict(stretch=1.0, original=0.0, low=1.0, high=32.0)
    args.update(kind)
    for rotary in (2, 64, 256):
        got = np.empty(rotary // 2)
        assert B.lib().dag_rope_frequencies(got.ctypes.data, rotary, args["theta"], args["stretch"], args["original"], args["low"], args["high"]) == 0
        want = q8.frequencies(rotary, **args)
        assert (np.abs(got - want) <= 2.0 ** -50 * want).all()
    got, f = np.empty(32), B.lib().dag_rope_frequencies
    assert f(None, 64, 1e4, 1.0, 0.0, 1.0, 32.0) == -1
    for bad in ((0, 1e4, 1.0, 0.0, 1.0, 32.0), (63, 1e4, 1.0, 0.0, 1.0, 32.0), (258, 1e4, 1.0, 0.0, 1.0, 32.0), (64, 0.0, 1.0, 0.0, 1.0, 32.0),
                (64, float("nan"), 1.0, 0.0, 1.0, 32.0), (64, float("inf"), 1.0, 0.0, 1.0, 32.0), (64, 1e4, 0.0, 0.0, 1.0, 32.0),
                (64, 1e4, float("nan"), 0.0, 1.0, 32.0), (64, 1e4, 1.0, -1.0, 1.0, 32.0), (64, 1e4, 1.0, 100.0, 4.0, 4.0),
                (64, 1e4, 1.0, 100.0, 4.0, float("nan"))):
        assert f(got.ctypes.data, *bad) == -7


def rows(n=4, page=16, width=8, pages=50, table=FAKE, free=FAKE):
    return C.byref(B.dag_kv_rows_t(n, page, width, pages, table, free))


FORK = (3,) + (FAKE,) * 12
RELEASE = (FAKE,) * 7
COMPACT = (FAKE,) * 8


@pytest.mark.parametrize("name,args,nullable", [("fork", FORK, (3, 12)), ("release_shared", RELEASE, ()), ("compact", COMPACT, ())])
def test_shared_pages(name, args, nullable):
    f, lib = getattr(B.lib(), "dag_kv_" + name), B.lib()
    need = lib.dag_kv_pages_workspace_bytes(4, 50, 3)
    assert need > 0 and lib.dag_kv_pages_workspace_bytes(-1, 50, 3) == 0 and lib.dag_kv_pages_workspace_bytes(4, -1, 3) == 0
    two = (lambda r: (r, r)) if name == "compact" else (lambda r: (r,))

    def call(r=None, a=args, ws=FAKE, size=need):
        return f(*two(r if r is not None else rows()), *a, ws, size, None)

    assert f(*((None, rows()) if name == "compact" else (None,)), *args, FAKE, need, None) == -1
    ints = [i for i, x in enumerate(args) if x == FAKE]
    for i in ints:
        if i not in nullable:
            assert call(a=replaced(args, i, 0)) == -1, i
    assert call(rows(page=32)) == -7 and call(rows(table=0)) == -1 and call(rows(free=0)) == -1
    for bad in (dict(n=-1), dict(width=-1), dict(pages=-1), dict(pages=2 ** 27), dict(width=2 ** 28)):
        assert call(rows(**bad)) == -2
    least = lib.dag_kv_pages_workspace_bytes(4, 50, 3 if name == "fork" else 0)
    assert call(ws=0) == -6 and call(size=least - 1) == -6 and call(ws=FAKE + 4) == -8
    if name == "fork":
        assert call(a=replaced(args, 0, -1)) == -2
    if name == "compact":
        assert f(rows(), None, *args, FAKE, need, None) == -1
        for bad in (dict(n=5), dict(width=9), dict(pages=51)):
            assert f(rows(), rows(**bad), *args, FAKE, need, None) == -2
        assert f(rows(), rows(page=8), *args, FAKE, need, None) == -7 and f(rows(), rows(table=0), *args, FAKE, need, None) == -1


def test_copies():
    f, g = B.lib().dag_kv_copy_pages_q8, B.lib().dag_kv_copy_pages
    assert f(None, FAKE, FAKE, 3, 0, None) == -1 and f(kv(), 0, FAKE, 3, 0, None) == -1 and f(kv(), FAKE, 0, 3, 0, None) == -1
    for name in ("k_pool", "v_pool", "k_scale", "v_scale"):
        assert f(kv(**{name: 0}), FAKE, FAKE, 3, 0, None) == -1 and f(kv(**{name: FAKE + 2}), FAKE, FAKE, 3, 0, None) == -8
    assert f(kv(), FAKE, FAKE, -1, 0, None) == -2 and f(kv(pages=-1), FAKE, FAKE, 3, 0, None) == -2
    assert f(kv(d=32), FAKE, FAKE, 3, 0, None) == -7 and f(kv(hkv=0), FAKE, FAKE, 3, 0, None) == -7
    assert f(kv(k_pool=0), 0, 0, 0, 0, None) == 0 and f(kv(pages=0), FAKE, FAKE, 3, 0, None) == 0
    ok = (FAKE, FAKE, 10, 2, 128, FAKE, FAKE, 3, 0, None)
    for i in (0, 1, 5, 6):
        assert g(*replaced(ok, i, 0)) == -1
    for i in (0, 1):
        assert g(*replaced(ok, i, FAKE + 8)) == -8
    assert g(*replaced(ok, 2, -1)) == -2 and g(*replaced(ok, 7, -1)) == -2 and g(*replaced(ok, 3, 0)) == -7 and g(*replaced(ok, 4, 96)) == -7


def test_binding():
    """Shapes and types are looked at before the library is called."""
    i32 = lambda n: torch.zeros(n, dtype=torch.int32)  # noqa: E731
    desc = B.PagedPrefillDesc.on_device(2, 4, 3, i32(3), i32(3), i32(6), i32(6), i32(2), i32(2))
    cache = B.KvCacheQ8.empty(5, 2, 64, "cpu")
    q, ws = torch.zeros((8, 4, 64), dtype=torch.bfloat16), torch.empty(256, dtype=torch.uint8)
    for bad in ((torch.zeros((8, 4, 32), dtype=torch.bfloat16), q), (q, q[:7]), (q.float(), q), (q.transpose(0, 1), q.transpose(0, 1)),
                (q, torch.zeros((8, 64, 4), dtype=torch.bfloat16).transpose(1, 2))):
        with pytest.raises((ValueError, TypeError)):
            B.dag_attn_prefill_paged_q8(desc, bad[0], cache, bad[1], ws)
    for lse in (torch.zeros((8, 4), dtype=torch.float64), torch.zeros((8, 5)), torch.zeros((4, 8)).t()):
        with pytest.raises(TypeError):
            B.dag_attn_prefill_paged_q8(desc, q, cache, q.clone(), ws, lse=lse)
    for bad in (dict(q_off=i32(2)), dict(own_len=i32(1)), dict(ctx_page_len=i32(5)), dict(own_page=torch.zeros(2))):
        args = dict(q_off=i32(3), ctx_page_off=i32(3), ctx_pages=i32(6), ctx_page_len=i32(6), own_page=i32(2), own_len=i32(2))
        args.update(bad)
        with pytest.raises((ValueError, TypeError)):
            B.PagedPrefillDesc.on_device(2, 4, 3, **args)
    r, x, pos = B.Rope(32, 1e4, "cpu"), torch.zeros((5, 3, 64)), i32(5)
    for bad in ((pos, x[:4], None), (pos, x.transpose(1, 2), None), (pos.long(), x, None), (pos, x, x.double()), (pos, x, torch.zeros((5, 3, 32))),
                (pos, x, None, x[:, :2])):
        with pytest.raises((ValueError, TypeError)):
            B.dag_rope_apply(r, *bad)
    with pytest.raises(ValueError):
        B.dag_rope_apply(r, pos, x, None, None, x)
    with pytest.raises(ValueError):
        B.Rope(32, 1e4, "cpu", freq=[1.0] * 15)
    with pytest.raises(B.DagError):
        B.Rope(33, 1e4, "cpu")
    k = torch.zeros((5, 2, 64))
    for bad in ((i32(5), i32(4), k, k), (i32(5), i32(5), k[:4], k), (i32(5), i32(5), k, k.to(torch.bfloat16)), (i32(5), i32(5), k, k.transpose(0, 1))):
        with pytest.raises((ValueError, TypeError)):
            B.dag_kv_append_rotary_q8(cache, *bad, r)
    t = B.KvRows(torch.zeros((3, 4), dtype=torch.int32), i32(9))
    with pytest.raises(ValueError):
        B.dag_kv_fork(t, i32(2), i32(1), i32(3), i32(3), i32(9), i32(9), i32(1), i32(1), i32(2), i32(2))
    with pytest.raises(ValueError):
        B.dag_kv_fork(t, i32(2), i32(2), i32(3), i32(3), i32(8), i32(9), i32(1), i32(1), i32(2), i32(2))
    with pytest.raises(ValueError):
        B.dag_kv_compact(t, t, i32(3), i32(9), i32(9), i32(1), i32(9), i32(3), i32(4), i32(1))
    with pytest.raises(ValueError):
        B.dag_kv_release_shared(t, i32(3), i32(3), i32(2), i32(9), i32(9), i32(1), i32(1))
    with pytest.raises(ValueError):
        B.dag_kv_copy_pages_q8(cache, i32(2), i32(3))
    pool = torch.zeros((4, 2, 64, 16), dtype=torch.bfloat16)
    with pytest.raises(ValueError):
        B.dag_kv_copy_pages(pool, pool, i32(2), i32(2))


def test_branches_are_refused():
    f = engine.Fork.__new__(engine.Fork)
    f.n, f.tokens, f.max_len = 3, 4, 10
    f.q, f.k = torch.zeros((3, 4, 64)), torch.zeros((3, 2, 64))
    good = [torch.zeros((3, 2, h, 64)) for h in (4, 2, 2)]
    for i, bad in ((0, good[0][:2]), (1, good[1][:, :1]), (2, good[2][..., :32]), (0, good[0][:, :, :2])):
        with pytest.raises(ValueError):
            f.extend(*[bad if j == i else x for j, x in enumerate(good)])
    with pytest.raises(ValueError, match="full"):
        f.extend(*[x.repeat(1, 4, 1, 1) for x in good])
    for parents in ([0, 1], [0, 0, 1], [0, 3, 2], [1, 1, -1]):
        with pytest.raises(ValueError):
            f.select(parents)

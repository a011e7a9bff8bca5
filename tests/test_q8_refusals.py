"""CPU: what the entry points of the 8-bit cache and of the page tables refuse, before any GPU work."""
import ctypes as C

import pytest
import torch

from paper_2602_07529_amd import binding as B

FAKE = 0x10000  # a non-null, 16-byte aligned "device pointer"; never dereferenced on these paths


def kv(pages=10, hkv=2, d=128, **other):
    f = dict(k_pool=FAKE, v_pool=FAKE, k_scale=FAKE, v_scale=FAKE)
    f.update(other)
    return C.byref(B.dag_kv_q8_t(f["k_pool"], f["v_pool"], f["k_scale"], f["v_scale"], pages, hkv, d))


def test_append():
    f = B.lib().dag_kv_append_rope_q8
    ok = (FAKE, FAKE, 5, FAKE, FAKE, 1e4, B.DAG_BF16, None)
    assert f(None, *ok) == -1
    for i in (0, 1, 3, 4):
        assert f(kv(), *(0 if j == i else x for j, x in enumerate(ok))) == -1
    for name in ("k_pool", "v_pool", "k_scale", "v_scale"):
        assert f(kv(**{name: 0}), *ok) == -1
        assert f(kv(**{name: FAKE + 2}), *ok) == -8
    for i in (3, 4):
        assert f(kv(), *(FAKE + 8 if j == i else x for j, x in enumerate(ok))) == -8
    assert f(kv(d=96), *ok) == -7 and f(kv(hkv=0), *ok) == -7 and f(kv(d=256), *ok) == -7
    assert f(kv(), FAKE, FAKE, 5, FAKE, FAKE, 0.0, B.DAG_BF16, None) == -7
    assert f(kv(), FAKE, FAKE, 5, FAKE, FAKE, float("nan"), B.DAG_BF16, None) == -7
    assert f(kv(), FAKE, FAKE, 5, FAKE, FAKE, 1e4, 2, None) == -7
    assert f(kv(), FAKE, FAKE, -1, FAKE, FAKE, 1e4, B.DAG_BF16, None) == -2
    assert f(kv(), FAKE, FAKE, 1 << 31, FAKE, FAKE, 1e4, B.DAG_BF16, None) == -2
    assert f(kv(pages=-1), *ok) == -2
    assert f(kv(k_pool=0), 0, 0, 0, 0, 0, 1e4, B.DAG_BF16, None) == 0  # nothing to store


def cascade(groups=2, live=4, page=16, shared=40, own=5, most=2, arrays=FAKE):
    return B.dag_decode_desc_t(groups, live, page, shared, own, most, *([arrays] * 8))


def segments(live=4, segs=3, page=16, pages=40, readers=4, total=6, arrays=FAKE):
    return B.dag_decode_seg_desc_t(live, segs, page, pages, readers, total, *([arrays] * 7), None)


@pytest.mark.parametrize("form", ["decode", "decode_segments"])
def test_attention(form):
    make = cascade if form == "decode" else segments
    need_of, f = getattr(B.lib(), "dag_%s_q8_workspace_bytes" % form), getattr(B.lib(), "dag_attn_%s_q8" % form)
    desc = make()
    need = need_of(C.byref(desc), 8, 2, 128)
    assert need >= 4 * 8 * (128 + 2) * 4
    ok = (FAKE, FAKE, 8, 0.1, FAKE, need, None)
    assert f(None, kv(), *ok) == -1 and f(C.byref(desc), None, *ok) == -1
    for i in (0, 1):
        assert f(C.byref(desc), kv(), *(0 if j == i else x for j, x in enumerate(ok))) == -1
        assert f(C.byref(desc), kv(), *(FAKE + 4 if j == i else x for j, x in enumerate(ok))) == -8
    for name in ("k_pool", "v_pool", "k_scale", "v_scale"):
        assert f(C.byref(desc), kv(**{name: 0}), *ok) == -1
        assert f(C.byref(desc), kv(**{name: FAKE + 2}), *ok) == -8
    assert f(C.byref(desc), kv(), FAKE, FAKE, 8, 0.1, FAKE, need - 1, None) == -6
    assert f(C.byref(desc), kv(), FAKE, FAKE, 8, 0.1, 0, need, None) == -6
    for hq in (7, 0, -8, 66):
        assert f(C.byref(desc), kv(), FAKE, FAKE, hq, 0.1, FAKE, need, None) == -7
        assert need_of(C.byref(desc), hq, 2, 128) == 0
    assert f(C.byref(desc), kv(d=32), *ok) == -7 and f(C.byref(desc), kv(hkv=0), *ok) == -7
    assert f(C.byref(desc), kv(pages=0), *ok) == -2 and f(C.byref(desc), kv(pages=-3), *ok) == -2
    assert f(C.byref(make(page=32)), kv(), *ok) == -7 and f(C.byref(make(live=-1)), kv(), *ok) == -2
    assert f(C.byref(make(arrays=0)), kv(), *ok) == -1
    assert f(C.byref(make(live=0)), kv(k_pool=0), 0, 0, 8, 0.1, 0, 0, None) == 0
    big = make(live=1 << 20, **({"own": 1 << 20} if form == "decode" else {"total": 1 << 28, "pages": 1 << 20}))
    assert f(C.byref(big), kv(), *ok) == -7 and need_of(C.byref(big), 8, 2, 128) == 0


def test_tables():
    L = B.lib()
    need = L.dag_kv_tables_workspace_bytes(5)
    assert need >= 40 and L.dag_kv_tables_workspace_bytes(-1) == 0

    def rows(n=5, page=16, width=8, pages=20, table=FAKE, free=FAKE):
        return C.byref(B.dag_kv_rows_t(n, page, width, pages, table, free))

    ok = (FAKE, FAKE, FAKE, FAKE, FAKE, FAKE, need, None)
    ok_t = (FAKE, FAKE, FAKE, FAKE, FAKE, FAKE, FAKE, 5, FAKE, FAKE, FAKE, FAKE, 20, FAKE, FAKE, need, None)
    for f, args, nullable, ws in ((L.dag_kv_release, ok, (), 5), (L.dag_kv_tables, ok_t, (8, 9, 11, 13), 14)):
        assert f(None, *args) == -1
        for i in range(ws):
            if i not in nullable and not (f is L.dag_kv_tables and i in (7, 12)):
                assert f(rows(), *(0 if j == i else x for j, x in enumerate(args))) == -1, i
        assert f(rows(), *(0 if j == ws else x for j, x in enumerate(args))) == -6
        assert f(rows(), *(FAKE + 2 if j == ws else x for j, x in enumerate(args))) == -8
        assert f(rows(), *(need - 1 if j == ws + 1 else x for j, x in enumerate(args))) == -6
        assert f(rows(page=32), *args) == -7
        for bad in (dict(n=-1), dict(width=-1), dict(pages=-1), dict(pages=1 << 27), dict(width=1 << 28)):
            assert f(rows(**bad), *args) == -2
        assert f(rows(table=0), *args) == -1 and f(rows(free=0), *args) == -1
    for i in (7, 12):
        assert L.dag_kv_tables(rows(), *(-1 if j == i else x for j, x in enumerate(ok_t))) == -2
        assert L.dag_kv_tables(rows(), *(1 << 31 if j == i else x for j, x in enumerate(ok_t))) == -2


def test_the_binding_looks_at_shapes_types_and_devices():
    e4, f32, i32 = torch.float8_e4m3fn, torch.float32, torch.int32
    k, v, s = torch.zeros(4, 2, 4, 16, 16).to(e4), torch.zeros(4, 2, 64, 16).to(e4), torch.ones(4, 2)
    cache = B.KvCacheQ8(k, v, s, s.clone())
    for bad in ((k[:3], v, s, s), (k, v.transpose(2, 3), s, s), (k, v, s[:, :1], s), (k, v, s, s.t().contiguous())):
        with pytest.raises(ValueError):
            B.KvCacheQ8(*bad)
    for bad in ((k.view(torch.uint8), v, s, s), (k, v, s.double(), s), (k, v, torch.ones(2, 4).t(), s)):
        with pytest.raises(TypeError):
            B.KvCacheQ8(*bad)
    n = torch.zeros(3, dtype=i32)
    x = torch.zeros(3, 2, 64, dtype=torch.bfloat16)
    for bad in ((n, n[:2], x, x), (n, n, x[:2], x), (n, n, x, x.float()), (n, n, x[:, :1], x), (n, n, torch.zeros(3, 64, 2, dtype=torch.bfloat16).transpose(1, 2), x)):
        with pytest.raises(ValueError):
            B.dag_kv_append_rope_q8(cache, *bad, 1e4)
    for bad in ((n.long(), n), (torch.zeros(6, dtype=i32)[::2], n)):
        with pytest.raises(TypeError):
            B.dag_kv_append_rope_q8(cache, *bad, x, x, 1e4)
    d = B.DecodeDesc.on_device(0, 3, 0, 2, 0, branch_page_off=torch.zeros(4, dtype=i32), branch_pages=n, branch_len=n)
    q = torch.zeros(3, 4, 64, dtype=torch.bfloat16)
    for bad in ((q[:2], q[:2]), (q[..., :32], q[..., :32]), (q, q[:2])):
        with pytest.raises(ValueError):
            B.dag_attn_decode_q8(d, bad[0], cache, bad[1], torch.zeros(9, dtype=torch.uint8))
    with pytest.raises(TypeError):
        B.dag_attn_decode_q8(d, q.float(), cache, q, torch.zeros(9, dtype=torch.uint8))
    with pytest.raises(TypeError):
        B.DecodeDesc.on_device(0, 3, 0, 2, 0, branch_page_off=torch.zeros(4), branch_pages=n, branch_len=n)
    rows = B.KvRows(torch.zeros(3, 5, dtype=i32), torch.zeros(7, dtype=i32))
    one, off = torch.zeros(1, dtype=i32), torch.zeros(4, dtype=i32)
    for bad in ((n[:2], n, n, one, one), (n, n, n, n, one), (n, n, off, one, one)):
        with pytest.raises(ValueError):
            B.dag_kv_release(rows, *bad)
    for bad in ((n, n, n, one, one, n, n), (n, off, n, one, one, off, n)):
        with pytest.raises(ValueError):
            B.dag_kv_tables(rows, *bad)
    with pytest.raises(ValueError):
        B.dag_kv_tables(rows, n, n, n, one, one, off, n, pos=one)


def test_descriptions_whose_arrays_are_too_short_or_on_several_devices():
    a = lambda n, device="cpu": torch.zeros(n, dtype=torch.int32, device=device)  # noqa: E731
    good = dict(group_branch_off=a(3), shared_page_off=a(3), shared_pages=a(1), shared_len=a(2), branch_page_off=a(5), branch_pages=a(1), branch_len=a(4))
    B.DecodeDesc.on_device(2, 4, 1, 1, 2, **good)
    B.DecodeDesc.on_device(0, 4, 0, 1, 0, **{k: v for k, v in good.items() if k[:6] == "branch"})
    for name in ("group_branch_off", "shared_page_off", "shared_len", "branch_page_off", "branch_len"):
        for bad in (a(good[name].numel() - 1), good[name].to("meta")):
            with pytest.raises(ValueError):
                B.DecodeDesc.on_device(2, 4, 1, 1, 2, **{**good, name: bad})
    good = dict(seg_page_off=a(4), seg_pages=a(1), seg_len=a(3), seg_reader_off=a(4), seg_readers=a(5), branch_entry_off=a(3), branch_entries=a(5),
                seg_reader_len=a(5))
    B.SegDecodeDesc.on_device(2, 3, 1, 2, 5, **good)
    for name in ("seg_page_off", "seg_len", "seg_reader_off", "branch_entry_off", "seg_reader_len"):
        for bad in (a(good[name].numel() - 1), good[name].to("meta")):
            with pytest.raises(ValueError):
                B.SegDecodeDesc.on_device(2, 3, 1, 2, 5, **{**good, name: bad})
    e4 = torch.zeros(4, 2, 4, 16, 16).to(torch.float8_e4m3fn), torch.zeros(4, 2, 64, 16).to(torch.float8_e4m3fn)
    with pytest.raises(ValueError):
        B.KvCacheQ8(*e4, torch.ones(4, 2), torch.ones(4, 2, device="meta"))
    with pytest.raises(ValueError):
        B.KvRows(a((3, 5)), a(7, "meta"))

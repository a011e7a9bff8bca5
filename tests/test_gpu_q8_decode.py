"""GPU: attention over the 8-bit cache, both forms of the description, against the oracle (tolerances: q8_cases)."""
import numpy as np
import pytest
import torch

from paper_2602_07529_amd import binding as B
from tests.gpu_util import DEV
from tests.q8_cases import Cascade, Segments, check, ints

pytestmark = pytest.mark.gpu

HEADS = [(1, 1, 64), (8, 2, 128), (5, 1, 128), (16, 8, 64), (12, 1, 128), (32, 1, 64), (34, 2, 128)]


def run(case, **kw):
    case.call(**kw)
    torch.cuda.synchronize()
    check(case.out, case.q, case.contexts, case.cache, kw.get("softmax_scale"))
    return case


# groups: one token; ends of pages, blocks of 32 and 64 keys; uneven siblings; long slices; nothing to share; nothing at all
GROUPS = {
    "one": [(0, [1])],
    "ends": [(n, [m, 1]) for n, m in ((15, 16), (16, 17), (17, 31), (31, 32), (32, 33), (33, 47), (48, 63), (64, 65), (65, 15))],
    "uneven": [(100, [3]), (0, [40, 7, 0]), (333, [1] * 9), (5, [200, 0])],
    "empty_rows": [(0, [0, 5, 0]), (20, [0, 0])],
    "long": [(5000, [700, 20, 333]), (2777, [16])],
    "many": [(70, [20] * 3)] * 30,
}


@pytest.mark.parametrize("groups", list(GROUPS))
@pytest.mark.parametrize("hq,hkv,d", HEADS)
def test_cascade(groups, hq, hkv, d):
    run(Cascade(GROUPS[groups], hq, hkv, d, seed=len(groups) + hq))


@pytest.mark.parametrize("hq,hkv,d,branches", [(8, 1, 128, 40), (40, 8, 128, 7), (10, 2, 64, 33), (4, 4, 128, 70)])
@pytest.mark.parametrize("shared", [37, 1500])
def test_groups_of_many_rows(hq, hkv, d, branches, shared):
    run(Cascade([(shared, [21] * branches), (shared // 2, [5] * (branches // 2))], hq, hkv, d, seed=shared))


@pytest.mark.parametrize("scales,spare,scale", [("any", 0, None), ("powers", 37, None), ("powers", 0, -0.05), ("any", 3, 1.7)])
def test_any_scale_bounds_above_the_lists_and_softmax_scales_of_either_sign(scales, spare, scale):
    kw = {} if scale is None else dict(softmax_scale=scale)
    run(Cascade([(200, [30, 50]), (1000, [3])], 8, 2, 128, 3, scales, spare), **kw)
    run(Segments(3, [(200, [(0, 200), (1, 70)]), (1000, [(2, 1000)]), (40, [(0, 9)])], 8, 2, 128, 3, scales, spare), **kw)


def test_scales_far_apart_in_one_context():
    c = Cascade([(160, [40, 18])], 8, 2, 128, 5)
    c.cache.v_scale.copy_(torch.exp2(torch.arange(c.cache.v_scale.numel(), device=DEV).reshape(c.cache.v_scale.shape) * 4.0 - 100))  # 2^-100 .. 2^16
    c.cache.k_scale.mul_(torch.exp2(torch.arange(c.cache.k_scale.shape[0], device=DEV)[:, None] % 5 - 2.0))
    run(c)


def test_large_scores_move_the_reference_at_every_block():
    c = Cascade([(640, [100, 333])], 8, 2, 128, 6)
    grow = torch.arange(c.cache.k_scale.shape[0], device=DEV, dtype=torch.float32)[:, None]
    c.cache.k_scale.copy_((2.0 ** -7) * (1 + grow / 4).expand_as(c.cache.k_scale))
    run(c)
    c.q.mul_(-1)
    run(c)


def test_no_group_and_page_ids_outside_the_pool_behind_the_lists():
    c = Cascade([(0, [33]), (0, [1]), (0, [200])], 8, 2, 64, 8)
    d = c.desc.t
    desc = B.DecodeDesc.on_device(0, 3, 50, 20, 5, branch_page_off=d["branch_page_off"], branch_pages=d["branch_pages"], branch_len=d["branch_len"])
    ws = torch.empty(max(256, B.dag_decode_q8_workspace_bytes(desc, c.cache, 8)), dtype=torch.uint8, device=DEV)
    d["branch_pages"][-1] = 2 ** 31 - 1
    B.dag_attn_decode_q8(desc, c.q, c.cache, c.out, ws)
    check(c.out, c.q, c.contexts, c.cache)
    d["branch_pages"][0] = -7  # a bad id inside a list: some page of the pool is read in its place, and the other rows are right
    B.dag_attn_decode_q8(desc, c.q, c.cache, c.out, ws)
    assert torch.isfinite(c.out[1:]).all()
    check(c.out, c.q, c.contexts, c.cache, rows=[1, 2])


def test_a_row_that_is_no_number_stays_by_itself():
    c = Cascade([(100, [20, 30, 5])], 8, 2, 128, 9)
    c.q[1, 3, 7] = float("nan")
    c.call()
    assert torch.isnan(c.out[1, 3]).all()
    c.out[1, 3] = 0
    keep = c.q.clone()
    c.q[1, 3] = 0
    good = c.out.clone()
    c.call()
    good[1, 3] = c.out[1, 3]
    assert torch.equal(good, c.out)
    c.q.copy_(keep)


SEGMENTS = {
    "one": (1, [(1, [(0, 1)])]),
    "levels": (6, [(300, [(r, 300) for r in range(6)]), (47, [(0, 47), (2, 47), (4, 47)]), (0, [(1, 0)]), (130, [(5, 130)])]
               + [(n, [(r, n)]) for r, n in enumerate((1, 15, 16, 17, 33, 64))]),
    "nothing": (4, [(20, [(1, 20)]), (5, []), (0, [(0, 0), (2, 0)])]),
    "limits": (5, [(100, [(0, 100), (1, 0), (2, 1), (3, 99), (4, 500)]), (33, [(0, 5), (1, 33), (3, -4), (4, 17)])]),
    "chunk": (40, [(700, [(r, 700) for r in range(40)]), (90, [(r, 51 + r) for r in range(40)])]),
    "long": (3, [(6000, [(0, 6000), (1, 100), (2, 3001)]), (77, [(1, 77)])]),
    "many": (60, [(100, [(r, 100) for r in range(20)])] + [(30 + r, [(r, 30 + r)]) for r in range(60)] + [(9, [(r, 9)]) for r in range(60)] * 3),
}


@pytest.mark.parametrize("segments", list(SEGMENTS))
@pytest.mark.parametrize("hq,hkv,d", HEADS)
def test_segments(segments, hq, hkv, d):
    n, segs = SEGMENTS[segments]
    limits = any(m < t for t, rs in segs for _, m in rs)
    run(Segments(n, segs, hq, hkv, d, seed=hq, limits=limits, shuffle=True, spare=2 if segments == "levels" else 0))


def test_values_that_are_no_number_reach_the_rows_that_see_them_and_no_others():
    n = 20
    c = Segments(n, [(200, [(r, 200) for r in range(n)]), (60, [(r, 41 + r) for r in range(n)])], 8, 2, 128, 4)
    page, slot = int(c.contexts[0][1][0][3]), 3  # token 51 of the second segment: rows 11 .. see it
    c.cache.v_pool.view(torch.uint8)[page, 1, 77, slot] = 0x7f
    c.call()
    bad = torch.isnan(c.out)
    want = torch.zeros_like(bad)
    want[11:, 4:, 77] = True
    assert torch.equal(bad, want)
    c.out[bad] = 0
    c.cache.v_pool.view(torch.uint8)[page, 1, 77, slot] = 0
    got = c.out.clone()
    c.call()
    c.out[want] = 0
    assert torch.equal(got, c.out)


def test_same_bits_on_any_stream_and_after_other_calls():
    c = Cascade([(700, [30] * 5), (90, [3])], 8, 2, 128, 11)
    s = Segments(4, [(300, [(r, 300) for r in range(4)]), (50, [(2, 50)])], 8, 2, 128, 12, limits=False)
    c.call()
    s.call()
    first = c.out.clone(), s.out.clone()
    torch.cuda.synchronize()
    with torch.cuda.stream(torch.cuda.Stream()):
        c.ws.fill_(0x7f)
        s.ws.fill_(0x7f)
        s.call()
        c.call()
        torch.cuda.current_stream().synchronize()
    assert torch.equal(c.out, first[0]) and torch.equal(s.out, first[1])


@pytest.mark.parametrize("form", ["cascade", "segments"])
def test_captured_and_replayed_with_lengths_that_change(form):
    if form == "cascade":
        c = Cascade([(200, [20, 33, 16]), (40, [5])], 8, 2, 128, 13, spare=1)
        lens = c.desc.t["branch_len"]
    else:
        c = Segments(4, [(200, [(r, 200) for r in range(4)])] + [(20 + r, [(r, 64)]) for r in range(4)], 8, 2, 128, 13)
        lens = c.desc.t["seg_len"]
    # (the slots that lengths grow into)
    c.cache.k_pool.view(torch.uint8).masked_fill_((c.cache.k_pool.view(torch.uint8) & 0x7f) == 0x7f, 0x30)
    c.cache.v_pool.view(torch.uint8).masked_fill_((c.cache.v_pool.view(torch.uint8) & 0x7f) == 0x7f, 0x30)
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        c.call()
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            c.call()
        for i in range(4):
            c.out.zero_()
            torch.cuda.synchronize()
            graph.replay()
            torch.cuda.synchronize()
            replayed = c.out.clone()
            c.out.zero_()
            c.call()
            torch.cuda.synchronize()
            assert torch.equal(c.out, replayed)
            lens[-1] += 1
    torch.cuda.synchronize()


def test_pool_offsets_past_32_bits():
    """Pages whose codes lie more than 4 GiB into the pools."""
    hkv, d = 8, 128
    n_pages = (5 << 30) // (hkv * d * 16)
    c = Cascade([(100, [20, 3])], 8, 8, 128, 14)
    far = {}
    for name in ("k_pool", "v_pool"):
        t = getattr(c.cache, name)
        far[name] = torch.zeros((n_pages,) + tuple(t.shape[1:]), dtype=torch.uint8, device=DEV).view(torch.float8_e4m3fn)
    for name in ("k_scale", "v_scale"):
        far[name] = torch.ones((n_pages, hkv), dtype=torch.float32, device=DEV)
    n = c.cache.k_scale.shape[0]
    for name, t in far.items():
        (t.view(torch.uint8) if "pool" in name else t)[-n:] = getattr(c.cache, name).view(torch.uint8) if "pool" in name else getattr(c.cache, name)
    c.call()
    want = c.out.clone()
    d = c.desc.t
    d["shared_pages"] += n_pages - n
    d["branch_pages"] += n_pages - n
    B.dag_attn_decode_q8(c.desc, c.q, B.KvCacheQ8(**far), c.out, c.ws)
    assert torch.equal(c.out, want)

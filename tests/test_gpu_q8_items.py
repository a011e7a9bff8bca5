"""GPU: steps over the 8-bit cache by work items, the route asserted: values that are no number, lengths that change under replay; what replayed
tables write for tokens and pages."""
import numpy as np
import pytest
import torch

from paper_2602_07529_amd import binding as B
from tests import q8_rules
from tests.gpu_util import DEV
from tests.q8_cases import Cascade, Segments, check, ints
from tests.test_gpu_q8_routes import replay_in_turn

pytestmark = pytest.mark.gpu


def _numbers(cache):
    """No code that is no number: for slots that lengths grow into."""
    for pool in (cache.k_pool, cache.v_pool):
        x = pool.view(torch.uint8)
        x.masked_fill_((x & 0x7f) == 0x7f, 0x30)


@pytest.mark.parametrize("hq,hkv,d", [(8, 2, 128), (20, 1, 64), (40, 2, 64), (4, 4, 128)])
@pytest.mark.parametrize("code", [0x7f, 0xff])
@pytest.mark.parametrize("token", [41, 47, 48, 52, 60, 63])
def test_a_value_that_is_no_number_reaches_the_rows_that_see_it_and_no_others(token, code, hq, hkv, d):
    n = 20
    sees = [40 + r * 7 % n + (r % 3) * 4 for r in range(n)]
    c = Segments(n, [(200, [(r, 200) for r in range(n)]), (70, list(enumerate(sees)))], hq, hkv, d, 51, spare=400)
    assert not q8_rules.segments_whole(c.desc.c, hkv, d)
    page, h, dim = int(c.contexts[0][1][0][token // 16]), hkv - 1, d - 3
    c.call()
    good = c.out.clone()
    was = int(c.cache.v_pool.view(torch.uint8)[page, h, dim, token % 16])
    c.cache.v_pool.view(torch.uint8)[page, h, dim, token % 16] = code
    c.call()
    torch.cuda.synchronize()
    want = torch.zeros_like(good, dtype=torch.bool)
    want[[r for r in range(n) if sees[r] > token], h * (hq // hkv):, dim] = True
    assert want.any() and torch.equal(torch.isnan(c.out), want)
    # the others: as with a value of nothing in its place, for the rows that see it in other dimensions nothing changes at all
    assert torch.equal(c.out[~want], good[~want])
    c.cache.v_pool.view(torch.uint8)[page, h, dim, token % 16] = was
    c.call()
    torch.cuda.synchronize()
    check(c.out, c.q, c.contexts, c.cache)


@pytest.mark.parametrize("form", ["cascade", "wide", "segments", "limits", "many"])
def test_captured_and_replayed_with_lengths_that_change(form):
    hkv, spare = 2, 400
    if form in ("cascade", "wide"):
        hq = 8 if form == "cascade" else 40
        c = Cascade([(900, [20, 33, 16]), (40, [5])], hq, hkv, 128, 52, spare=spare)
        assert not q8_rules.plan(c.desc.c, hq, hkv, 128).whole
        lens = [("branch_len", -1, lambda n: c.contexts[-1].__setitem__(1, (c.contexts[-1][1][0], n))),
                ("shared_len", 0, lambda n: [x.__setitem__(0, (x[0][0], n)) for x in c.contexts[:3]])]
        steps = [(5, 900), (6, 880), (16, 1), (0, 0), (11, 897), (1, 16)]
    else:
        hq, n = 8, 4
        many = form == "many"  # (more segments than a workgroup of the plan has threads)
        segs = [(900, [(r, 900) for r in range(n)])] + [(5 + r, [(r, 64)]) for r in range(n)] + [(3, [(i % n, 3)]) for i in range(1100 * many)]
        c = Segments(n, segs, hq, hkv, 128, 53, spare=spare, limits=form == "limits")
        assert not q8_rules.segments_whole(c.desc.c, hkv, 128)
        lens = [("seg_len", 4, lambda n: c.contexts[-1].__setitem__(1, (c.contexts[-1][1][0], n))),
                ("seg_len", 0, lambda n: [x.__setitem__(0, (x[0][0], n)) for x in c.contexts])]
        steps = [(8, 900), (9, 300), (16, 17), (0, 0), (12, 897), (1, 1)]
    _numbers(c.cache)
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        c.call()
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            c.call()
        for step in steps:
            for (name, at, note), value in zip(lens, step):
                c.desc.t[name][at] = value
                note(value)
            c.out.fill_(float("nan"))
            graph.replay()
            torch.cuda.synchronize()
            replayed = c.out.clone()
            c.out.fill_(float("nan"))
            c.ws.fill_(0xff)
            c.call()
            torch.cuda.synchronize()
            assert torch.equal(c.out, replayed)
            check(c.out, c.q, c.contexts, c.cache)


@pytest.mark.parametrize("n_rows", [5, 1024, 1500])
def test_slots_and_pages_of_graphs_that_share_rows(n_rows):
    rng = np.random.default_rng(n_rows)
    lens, width, n_pages = rng.integers(0, 60, n_rows), 8, 12 * n_rows
    perm = rng.permutation(n_pages).astype(np.int32)
    rows = B.KvRows(ints(perm[:n_rows * width]).reshape(n_rows, width), ints(perm))
    outs, calls = [], []
    for most in (1, 40):
        new, ended = ints(rng.integers(0, most + 1, n_rows)), ints(rng.integers(0, 2, n_rows))
        z = lambda n: torch.zeros(n, dtype=torch.int32, device=DEV)  # noqa: E731
        old, count, pos0 = ints(lens), ints([4 * n_rows]), ints(rng.integers(0, 1000, n_rows))
        o = dict(l1=z(n_rows), c1=z(1), l2=z(n_rows), c2=z(1), off=z(n_rows + 1), slots=z(n_rows * most), pos=z(n_rows * most),
                 page_off=z(n_rows + 1), pages=z(n_rows * width), refused=z(1))

        def call(o=o, new=new, ended=ended, old=old, count=count, pos0=pos0):
            B.dag_kv_tables(rows, new, old, o["l2"], count, o["c2"], o["off"], o["slots"], pos0=pos0, pos=o["pos"], page_off=o["page_off"],
                            pages=o["pages"], refused=o["refused"])
            B.dag_kv_release(rows, ended, old, o["l1"], count, o["c1"])

        calls.append(call)
        outs.append([o[k] for k in ("slots", "pos", "pages", "l1", "l2", "off", "page_off")])
    replay_in_turn(calls, outs)
    assert all(int(x[0].abs().sum()) > 0 for x in outs)

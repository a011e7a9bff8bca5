"""GPU: the same steps over an 8-bit cache by one launch and by work items (the host bounds above the lists decide), against the oracle; what
captured graphs may share."""
import numpy as np
import pytest
import torch

from paper_2602_07529_amd import binding as B
from tests import q8_rules
from tests.gpu_util import DEV
from tests.q8_cases import Cascade, Segments, check, ints

pytestmark = pytest.mark.gpu

STEPS = {
    "one": ([(0, [1])], 4, 1),
    "ends": ([(16, [16, 17]), (33, [1, 15]), (0, [32])], 8, 2),
    "prefix": ([(480, [100, 3, 77])], 32, 8),
    "odd": ([(77, [50] * 5), (200, [0, 9])], 15, 3),
    "tall": ([(64, [33] * 9)], 32, 1),
    "full": ([(300, [100] * 4)] * 8, 24, 8),
}


@pytest.mark.parametrize("whole", [True, False])
@pytest.mark.parametrize("step", list(STEPS))
@pytest.mark.parametrize("d", [64, 128])
def test_both_routes_of_a_cascade(step, d, whole):
    groups, hq, hkv = STEPS[step]
    c = Cascade(groups, hq, hkv, d, 21, spare=0 if whole else 120)
    assert bool(q8_rules.plan(c.desc.c, hq, hkv, d).whole) is whole
    c.call()
    torch.cuda.synchronize()
    check(c.out, c.q, c.contexts, c.cache)


@pytest.mark.parametrize("whole", [True, False])
@pytest.mark.parametrize("hq,hkv,d", [(4, 1, 64), (32, 8, 128), (15, 3, 128), (32, 1, 64)])
@pytest.mark.parametrize("limits", [True, False])
def test_both_routes_of_segments(hq, hkv, d, limits, whole):
    segs = [(400, [(r, 400 - 130 * limits * (r % 2)) for r in range(5)]), (0, [(2, 0)]), (47, [(1, 47), (3, 16 if limits else 47)])]
    segs += [(n, [(r, n)]) for r, n in enumerate((1, 16, 17, 32, 63))]
    c = Segments(5, segs, hq, hkv, d, 22, spare=0 if whole else 400, limits=limits, shuffle=True)
    assert q8_rules.segments_whole(c.desc.c, hkv, d) is whole
    c.call()
    torch.cuda.synchronize()
    check(c.out, c.q, c.contexts, c.cache)


def test_a_segment_without_readers_beside_the_most_that_one_launch_takes():
    segs = [(20, [(i % 7, 20)]) if i % 3 else (9, []) for i in range(64)]
    for n in (64, 65):
        c = Segments(7, segs + [(5, [(0, 5)])] * (n - 64), 8, 2, 128, 23, shuffle=True)
        assert q8_rules.segments_whole(c.desc.c, 2, 128) is (n == 64)
        c.call()
        torch.cuda.synchronize()
        check(c.out, c.q, c.contexts, c.cache)


def replay_in_turn(calls, outs):
    """Each call captured in a graph of its own; replays in turn, with eager calls between them, give what the eager calls give."""
    stream = torch.cuda.Stream()
    graphs = []
    with torch.cuda.stream(stream):
        want = []
        for call, out in zip(calls, outs):
            call()
            torch.cuda.synchronize()
            want.append([x.clone() for x in out])
        for call in calls:
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph, stream=stream):
                call()
            graphs.append(graph)
        for _ in range(3):
            for graph, call in zip(graphs, calls[::-1]):
                call()
                graph.replay()
            stream.synchronize()
            for w, out in zip(want, outs):
                assert all(torch.equal(a, b) for a, b in zip(w, out))
                for x in out:
                    x.fill_(0)
            for graph in graphs:
                graph.replay()
            stream.synchronize()
            for w, out in zip(want, outs):
                assert all(torch.equal(a, b) for a, b in zip(w, out))


def test_graphs_that_share_a_workspace_in_the_order_of_a_stream():
    a = Cascade([(3000, [200] * 4)], 8, 2, 128, 24)
    b = Segments(5, [(2500, [(r, 2500) for r in range(5)])] + [(300, [(r, 300 - r)]) for r in range(5)], 8, 2, 128, 25)
    c = Cascade([(100, [20] * 4)], 8, 2, 128, 26)
    ws = a.ws if a.ws.numel() > b.ws.numel() else b.ws
    a.ws = b.ws = c.ws = ws
    replay_in_turn([a.call, b.call, c.call], [[a.out], [b.out], [c.out]])


@pytest.mark.parametrize("n_rows", [5, 1024, 1500])
def test_tables_of_graphs_that_share_rows(n_rows):
    rng = np.random.default_rng(n_rows)
    lens, width, n_pages = rng.integers(0, 60, n_rows), 8, 12 * n_rows
    perm = rng.permutation(n_pages).astype(np.int32)
    rows = B.KvRows(ints(perm[:n_rows * width]).reshape(n_rows, width), ints(perm))
    outs, calls = [], []
    for most in (1, 40):
        new, ended = ints(rng.integers(0, most + 1, n_rows)), ints(rng.integers(0, 2, n_rows))
        z = lambda n: torch.zeros(n, dtype=torch.int32, device=DEV)  # noqa: E731
        old, count = ints(lens), ints([4 * n_rows])
        o = dict(l1=z(n_rows), c1=z(1), l2=z(n_rows), c2=z(1), off=z(n_rows + 1), slots=z(n_rows * most), page_off=z(n_rows + 1),
                 pages=z(n_rows * width), refused=z(1))

        def call(o=o, new=new, ended=ended, old=old, count=count):
            B.dag_kv_tables(rows, new, old, o["l2"], count, o["c2"], o["off"], o["slots"], page_off=o["page_off"], pages=o["pages"], refused=o["refused"])
            B.dag_kv_release(rows, ended, old, o["l1"], count, o["c1"])

        calls.append(call)
        outs.append([o[k] for k in ("l1", "c1", "l2", "c2", "off", "page_off", "refused")])
    replay_in_turn(calls, outs)
    assert int(rows.workspace[:4].sum()) == 0


@pytest.mark.parametrize("scale", [0.0, -0.0, 1e-30])
@pytest.mark.parametrize("spare", [0, 400])
def test_a_softmax_scale_of_nothing_gives_the_mean(scale, spare):
    c = Cascade([(70, [20, 33]), (0, [0, 1])], 8, 2, 128, 27, spare=spare)
    s = Segments(4, [(200, [(r, 200 - 50 * r) for r in range(4)]), (9, [(2, 9)])], 8, 2, 64, 28, spare=spare)
    for x in (c, s):
        x.call(softmax_scale=scale)
        torch.cuda.synchronize()
        check(x.out, x.q, x.contexts, x.cache, scale)


@pytest.mark.parametrize("hq,hkv,d", [(4, 1, 128), (16, 2, 64)])
def test_one_branch_over_a_very_long_context(hq, hkv, d):
    """Hundreds of partial results to a row, more than a merging wave takes at a time."""
    c = Cascade([(60001, [5])], hq, hkv, d, 29)
    assert q8_rules.plan(c.desc.c, hq, hkv, d).splits_a > 64
    s = Segments(2, [(60001, [(0, 60001), (1, 33333)]), (5, [(0, 5)])], hq, hkv, d, 30)
    for x in (c, s):
        x.call()
        torch.cuda.synchronize()
        check(x.out, x.q, x.contexts, x.cache)


def test_calls_at_once_on_two_streams_with_a_workspace_each():
    a = Cascade([(4000, [300] * 6)], 8, 2, 128, 31)
    b = Segments(6, [(3000, [(r, 3000) for r in range(6)])] + [(100, [(r, 100)]) for r in range(6)], 8, 2, 128, 32, limits=False)
    a.call()
    b.call()
    torch.cuda.synchronize()
    want = a.out.clone(), b.out.clone()
    streams = torch.cuda.Stream(), torch.cuda.Stream()
    for _ in range(4):
        a.out.zero_()
        b.out.zero_()
        torch.cuda.synchronize()
        for stream, x in zip(streams, (a, b)):
            with torch.cuda.stream(stream):
                for _ in range(3):
                    x.call()
        torch.cuda.synchronize()
        assert torch.equal(a.out, want[0]) and torch.equal(b.out, want[1])

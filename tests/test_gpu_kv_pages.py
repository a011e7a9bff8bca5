"""dag_kv_fork, dag_kv_release_shared, dag_kv_compact and the copies of pages against the oracle (equal to the bit)."""
import numpy as np
import pytest
import torch

from oracle import q8_oracle as q8
from paper_2602_07529_amd import binding as B
from tests.gpu_util import DEV
from tests.q8_cases import ints

pytestmark = pytest.mark.gpu


class Family:
    """A table of rows that own their pages, with the same in numpy beside it."""

    def __init__(self, lens, width, free, seed=0):
        rng = np.random.default_rng(seed)
        held = [min(-(-max(n, 0) // 16), width) for n in lens]
        n_pages = sum(held) + free
        perm = rng.permutation(n_pages).astype(np.int32)
        self.table = np.full((len(lens), width), -7, dtype=np.int32)
        at = 0
        for r, h in enumerate(held):
            self.table[r, :h] = perm[at:at + h]
            at += h
        self.free = np.full(n_pages, -9, dtype=np.int32)
        self.free[:free] = perm[at:]
        self.count, self.row_len, self.extra = free, np.asarray(lens, dtype=np.int32), np.zeros(n_pages, dtype=np.int32)
        self.upload()

    def upload(self):
        table = torch.from_numpy(self.table.copy()).to(DEV)
        self.rows = B.KvRows(table, torch.from_numpy(self.free.copy()).to(DEV))
        self.d_len, self.d_extra, self.d_count = ints(self.row_len), ints(self.extra), ints([self.count])

    def same(self):
        assert np.array_equal(self.rows.table.cpu().numpy(), self.table)
        assert np.array_equal(self.rows.free_pages.cpu().numpy(), self.free)
        assert np.array_equal(self.d_len.cpu().numpy(), np.maximum(self.row_len, 0))
        assert np.array_equal(self.d_extra.cpu().numpy(), self.extra)
        assert int(self.d_count) == self.count

    def fork(self, parent, child, fork_len=None, in_place=True):
        n = len(parent)
        src, dst, refused = ints([5] * n), ints([5] * n), ints([5])
        out = (self.d_len, self.d_extra, self.d_count) if in_place else (ints([3] * len(self.row_len)), ints([3] * len(self.extra)), ints([3]))
        B.dag_kv_fork(self.rows, ints(parent), ints(child), self.d_len, out[0], self.d_extra, out[1], self.d_count, out[2], src, dst,
                      None if fork_len is None else ints(fork_len), refused)
        self.d_len, self.d_extra, self.d_count = out
        self.count, s, d, bad = q8.fork(self.table, self.free, self.count, self.row_len, self.extra, parent, child, fork_len)
        assert src.tolist() == list(s) and dst.tolist() == list(d) and int(refused) == bad
        self.same()
        return s, d

    def release(self, ended, in_place=True):
        out = (self.d_len, self.d_extra, self.d_count) if in_place else (ints([3] * len(self.row_len)), ints([3] * len(self.extra)), ints([3]))
        B.dag_kv_release_shared(self.rows, ints(ended), self.d_len, out[0], self.d_extra, out[1], self.d_count, out[2])
        self.d_len, self.d_extra, self.d_count = out
        self.count = q8.release_shared(self.table, self.free, self.count, self.row_len, self.extra, ended)
        self.same()

    def compact(self, in_place=True):
        n = len(self.extra)
        to = self.rows if in_place else B.KvRows(self.rows.table.clone(), self.rows.free_pages.clone())
        extra = self.d_extra if in_place else ints([3] * n)
        page_map, src, dst, moved = ints([3] * n), ints([-3] * (n // 2)), ints([-3] * (n // 2)), ints([3])
        B.dag_kv_compact(self.rows, to, self.d_len, self.d_extra, extra, self.d_count, page_map, src, dst, moved)
        self.table, self.free, holders, new, pairs = q8.compact(self.table, self.free, self.count, self.row_len, self.extra)
        self.extra = holders.astype(np.int32)
        self.rows, self.d_extra = to, extra
        k = len(pairs)
        assert int(moved) == k and page_map.tolist() == new
        assert src.tolist() == [p for p, _ in pairs] + [-3] * (n // 2 - k) and dst.tolist() == [p for _, p in pairs] + [-3] * (n // 2 - k)
        self.same()
        return pairs


@pytest.mark.parametrize("in_place", [True, False])
def test_forks(in_place):
    f = Family([33, 0, 16, 0, 0, 0, 1, 0, 0, 160], 10, 9)
    f.fork([0, 0, 2, 9, 6, 1], [1, 3, 4, 5, 7, 8], in_place=in_place)
    f = Family([33, 0, 16, 0, 0, 0, 1, 0, 0, 160], 10, 9)
    f.fork([0, 0, 9, 9, 6], [1, 3, 4, 5, 7], [32, 17, 200, 0, -4], in_place)


def test_forks_that_are_refused():
    """Children that hold tokens, the same child twice, rows outside the table, too few pages; a parent that is a child too."""
    f = Family([33, 0, 20, 0, 0, 0, 17, 0, 0], 10, 2, seed=1)
    f.fork([0, 2, 0, 0, -1, 2, 99, 6, 3, 0, 2], [1, 1, 2, 3, 4, 9, 5, 4, 5, 7, 8])
    f = Family([48, 0, 0, 33, 0], 3, 0, seed=2)
    f.fork([0, 3, 0], [1, 2, 4])
    f = Family([-5, 0, 40], 3, 1, seed=2)
    f.fork([0, 2], [0, 1], in_place=False)


def test_no_forks_and_no_rows():
    f = Family([33, 0], 10, 3)
    f.fork([], [])
    f.fork([], [], in_place=False)
    f.compact()
    f.release([0, 0])
    empty = Family([], 4, 3)
    empty.fork([], [])
    empty.release([])
    empty.compact()


@pytest.mark.parametrize("rows,width,in_place", [(40, 9, True), (40, 9, False), (1500, 13, True), (3000, 40, False), (2, 300, True), (5000, 3, True), (4500, 2, False), (600, 5, True)])
def test_families(rows, width, in_place):
    """Forks of forks, releases and compactions behind one another, small tables (one workgroup) and large ones."""
    rng = np.random.default_rng(rows)
    lens = [int(rng.integers(1, width * 16 + 1)) if rng.random() < 0.4 else 0 for _ in range(rows)]
    f = Family(lens, width, rows // 3, seed=rows)
    for step in range(4):
        held, none = np.flatnonzero(f.row_len > 0), np.flatnonzero(f.row_len == 0)
        n = min(len(none), 2 * len(held), 1200)
        if n and len(held):
            child = rng.permutation(none)[:n]
            f.fork(rng.choice(held, n).tolist(), child.tolist(), [int(x) for x in rng.integers(0, width * 16, n)] if step % 2 else None, in_place)
        f.release((rng.random(rows) < 0.4).astype(int).tolist(), in_place)
        f.compact(in_place)
    f.release([1] * rows, in_place)
    assert f.count == len(f.extra) and not f.extra.any()


def test_page_ids_outside_the_pool():
    f = Family([40, 0, 20], 4, 5, seed=3)
    f.table[0, 0], f.table[0, 1] = -1, 10 ** 6
    f.upload()
    f.fork([0], [1])
    f.release([1, 1, 0])
    f.compact()


@pytest.mark.parametrize("hkv,d", [(1, 64), (8, 128), (3, 128)])
@pytest.mark.parametrize("bf16", [False, True])
def test_copies(hkv, d, bf16):
    rng = np.random.default_rng(hkv)
    n = 50
    perm = rng.permutation(n)
    src, dst = [int(x) for x in perm[:21]], [int(x) for x in perm[21:42]]
    src[3], dst[5], src[6] = -1, n, 2 ** 31 - 1
    if bf16:
        k, v = (torch.randn(s, device=DEV).to(torch.bfloat16) for s in ((n, hkv, d // 8, 16, 8), (n, hkv, d, 16)))
        arrays = [k, v]
        call = lambda *a, **kw: B.dag_kv_copy_pages(k, v, *a, **kw)  # noqa: E731
    else:
        cache = B.KvCacheQ8.empty(n, hkv, d, DEV)
        arrays = [cache.k_pool.view(torch.uint8), cache.v_pool.view(torch.uint8), cache.k_scale, cache.v_scale]
        for x in arrays[:2]:
            x.random_(0, 256)
        for x in arrays[2:]:
            x.uniform_()
        call = lambda *a, **kw: B.dag_kv_copy_pages_q8(cache, *a, **kw)  # noqa: E731
    for count in (None, 0, 7, 100):
        want = [x.clone() for x in arrays]
        for i, (s, t) in enumerate(zip(src, dst)):
            if 0 <= s < n and 0 <= t < n and (count is None or i < count):
                for x in want:
                    x[t] = x[s]
        call(ints(src), ints(dst), **({} if count is None else dict(count=ints([count]))))
        assert all(torch.equal(x, y) for x, y in zip(arrays, want))


def test_captured_steps():
    """A fork, a release and a compaction captured once; every replay goes on from the one in front."""
    f = Family([50, 0, 33, 0, 0, 0], 8, 30, seed=5)
    n, parent, child, ended = len(f.extra), [0, 0, 2], [1, 3, 4], [0, 1, 0, 1, 1, 0]
    src, dst, refused, page_map = ints([0] * 3), ints([0] * 3), ints([0]), ints([0] * n)
    m_src, m_dst, moved = ints([0] * (n // 2)), ints([0] * (n // 2)), ints([0])
    d_parent, d_child, d_ended = ints(parent), ints(child), ints(ended)
    cache = B.KvCacheQ8.empty(n, 2, 64, DEV)
    cache.v_scale.copy_(torch.arange(2 * n, device=DEV).reshape(n, 2))
    scales = cache.v_scale.cpu().numpy().copy()
    f.rows.for_shared()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        B.dag_kv_fork(f.rows, d_parent, d_child, f.d_len, f.d_len, f.d_extra, f.d_extra, f.d_count, f.d_count, src, dst, refused=refused)
        B.dag_kv_copy_pages_q8(cache, src, dst)
        B.dag_kv_release_shared(f.rows, d_ended, f.d_len, f.d_len, f.d_extra, f.d_extra, f.d_count, f.d_count)
        B.dag_kv_compact(f.rows, f.rows, f.d_len, f.d_extra, f.d_extra, f.d_count, page_map, m_src, m_dst, moved)
        B.dag_kv_copy_pages_q8(cache, m_src, m_dst, count=moved)
    for _ in range(4):
        graph.replay()
        torch.cuda.synchronize()
        f.count, s, d, bad = q8.fork(f.table, f.free, f.count, f.row_len, f.extra, parent, child, None)
        assert src.tolist() == list(s) and dst.tolist() == list(d) and int(refused) == bad
        for p, q in zip(s, d):
            if p >= 0:
                scales[q] = scales[p]
        f.count = q8.release_shared(f.table, f.free, f.count, f.row_len, f.extra, ended)
        f.table, f.free, holders, _, pairs = q8.compact(f.table, f.free, f.count, f.row_len, f.extra)
        for p, q in pairs:
            scales[q] = scales[p]
        f.extra = holders.astype(np.int32)
        f.same()
        assert np.array_equal(cache.v_scale.cpu().numpy(), scales)

"""GPU: dag_kv_release and dag_kv_tables against the oracle, row by row; whole numbers, so everything has to be equal."""
import numpy as np
import pytest
import torch

from oracle import q8_oracle as q8
from paper_2602_07529_amd import binding as B
from tests.gpu_util import DEV

pytestmark = pytest.mark.gpu

PAGE = 16


def ints(x):
    return torch.tensor(np.asarray(x, dtype=np.int32), device=DEV)


class Book:
    def __init__(self, lens, width, n_free, seed=0):
        rng = np.random.default_rng(seed)
        held = [min(-(-n // PAGE), width) for n in lens]
        n_pages = sum(held) + n_free
        perm = rng.permutation(n_pages).astype(np.int32)
        self.table = np.full((len(lens), width), -1, dtype=np.int32)
        at = 0
        for r, n in enumerate(held):
            self.table[r, :n] = perm[at:at + n]
            at += n
        self.free = np.full(n_pages, -1, dtype=np.int32)
        self.free[:n_free] = perm[at:]
        self.count, self.lens = n_free, np.asarray(lens, dtype=np.int64)
        self.pos0 = rng.integers(0, 1000, len(lens))
        self.d = dict(table=ints(self.table), free=ints(self.free), count=ints([n_free]), lens=ints(lens), pos0=ints(self.pos0))
        self.rows = B.KvRows(self.d["table"], self.d["free"])

    def same(self, lens, count):
        assert lens.cpu().tolist() == list(self.lens) and count.item() == self.count
        assert np.array_equal(self.d["table"].cpu().numpy(), self.table) and np.array_equal(self.d["free"].cpu().numpy(), self.free)

    def release(self, ended, in_place=True):
        d = self.d
        lens, count = (d["lens"], d["count"]) if in_place else (torch.empty_like(d["lens"]), torch.empty_like(d["count"]))
        B.dag_kv_release(self.rows, ints(ended), d["lens"], lens, d["count"], count)
        self.count = q8.release(self.table, self.free, self.count, self.lens, ended)
        self.same(lens, count)
        d["lens"], d["count"] = lens, count

    def extend(self, new, in_place=True, short=0, lists=True):
        """short: how many entries the lists are too short by."""
        d = self.d
        lens, count = (d["lens"], d["count"]) if in_place else (torch.empty_like(d["lens"]), torch.empty_like(d["count"]))
        n = len(new)
        total = max(0, int(sum(max(x, 0) for x in new)) - short)
        new_off, page_off, refused = ints(np.full(n + 1, -9)), ints(np.full(n + 1, -9)), ints([-9])
        slots, pos, pages = ints(np.full(total + 5, -9)), ints(np.full(total + 5, -9)), ints(np.full(len(self.free) + 5, -9))
        cap = max(0, len(self.free) - short)
        more = dict(pos0=d["pos0"], pos=pos[:total], page_off=page_off, pages=pages[:cap], refused=refused) if lists else {}
        B.dag_kv_tables(self.rows, ints(new), d["lens"], lens, d["count"], count, new_off, slots[:total], **more)
        left, off, s, p, poff, pg, no = q8.extend(self.table, self.free, self.count, self.lens, new, self.pos0)
        self.count = left
        self.same(lens, count)
        assert new_off.cpu().tolist() == off
        assert slots.cpu().tolist() == s[:total] + [-9] * (5 + max(0, total - len(s)))
        if lists:
            assert pos.cpu().tolist() == p[:total] + [-9] * 5
            assert page_off.cpu().tolist() == poff and refused.item() == no
            assert pages.cpu().tolist() == (pg[:cap] + [-9] * (len(pages) - len(pg[:cap])))
        d["lens"], d["count"] = lens, count
        return no


@pytest.mark.parametrize("in_place", [True, False])
@pytest.mark.parametrize("n_rows,old,new", [(1, 0, 1), (1, 15, 1), (1, 16, 1), (1, 5, 3000), (7, 100, 40), (64, 300, 1), (200, 31, 2), (1024, 90, 1),
                                            (1025, 40, 20), (2500, 20, 3), (1024, 60, 1), (1025, 60, 1),
                                            (1024, 1500, 900), (257, 1500, 900),
                                            (5000, 40, 3), (4096, 40, 3), (4097, 40, 20), (9000, 20, 3), (3, 5, 40000), (40, 3000, 1), (30, 9000, 700)])
def test_rows_grow_and_end(in_place, n_rows, old, new):
    rng = np.random.default_rng(n_rows + new)
    lens = rng.integers(0, old + 1, n_rows)
    width = -(-(old + 3 * new) // PAGE) + 1
    b = Book(lens, width, int(sum(-(-(n + 3 * new) // PAGE) for n in lens)))
    for step in range(3):
        b.extend(rng.integers(0, new + 1, n_rows) if new > 1 else np.ones(n_rows, dtype=np.int64), in_place)
        b.release(rng.random(n_rows) < (0.3, 1.0, 0.0)[step], in_place)


@pytest.mark.parametrize("n_rows", [1, 5, 300, 1500])
def test_pages_run_out_and_lines_are_full(n_rows):
    rng = np.random.default_rng(n_rows)
    lens = rng.integers(0, 200, n_rows)
    b = Book(lens, 13, n_rows * 2)
    assert sum(b.extend(rng.integers(0, 150, n_rows)) for _ in range(3)) > 0 or n_rows == 1
    assert b.extend(np.full(n_rows, 14 * PAGE)) == n_rows
    b.release(np.ones(n_rows))
    b.extend(np.full(n_rows, 20))


def test_nothing_at_all():
    b = Book([0, 0, 5], 3, 4)
    b.extend([0, 0, 0])
    b.release([0, 0, 0])
    b.release([1, 1, 0])
    b = Book([], 3, 4)
    b.extend([])
    b.release([])
    b = Book([0, 0], 0, 3)  # rows without room for a page
    assert b.extend([1, 0]) == 1
    b = Book([3, 0], 2, 0)  # no free page
    assert b.extend([13, 1]) == 1


def test_lists_shorter_than_needed_and_none_at_all():
    b = Book([40, 3, 100], 20, 40)
    b.extend([30, 0, 17], short=20)
    b.extend([5, 5, 5], short=100)
    b.extend([5, 5, 100], lists=False)


def test_negative_lengths_count_as_none():
    b = Book([40, 3], 20, 40)
    b.extend([-5, 4])
    b.d["lens"][1] = -3
    b.lens[1] = 0
    b.table[1, :] = b.d["table"][1].cpu().numpy()
    b.extend([1, 1])
    b.d["count"][0] = -2
    b.count = 0
    assert b.extend([20, 20]) == 2


def test_same_row_order_on_another_stream():
    got = []
    for stream in (torch.cuda.current_stream(), torch.cuda.Stream()):
        with torch.cuda.stream(stream):
            b = Book(np.arange(400), 60, 4000)
            b.extend(np.arange(400) % 37)
            b.release(np.arange(400) % 5 == 0)
            b.extend(np.arange(400) % 23)
            got.append((b.d["table"].cpu(), b.d["free"].cpu()))
    assert all(torch.equal(x, y) for x, y in zip(*got))

"""Page tables on the GPU against the oracle's lists: every table, count, list and pool byte after every call, exactly."""
import random

import numpy as np
import pytest
import torch

from oracle import kv4_oracle as O
from paper_2609_23900_b200 import binding
from tests.harness import ctx

pytestmark = pytest.mark.gpu


def i32(a):
    return torch.tensor(a, dtype=torch.int32, device="cuda")


class Both:
    """The same calls on both sides."""

    def __init__(self, n_rows, max_pages, n_pages, P, n_pools=2, page_bytes=48, seed=0):
        rs = np.random.default_rng(seed)
        host = [rs.integers(0, 256, (n_pages, page_bytes), dtype=np.uint8) for _ in range(n_pools)]
        self.o = O.Pages(n_rows, max_pages, n_pages, P, host)
        z = lambda *s: torch.full(s, -7, dtype=torch.int32, device="cuda")                    # noqa: E731
        self.t = dict(table=z(n_rows, max_pages), row_pages=z(n_rows), refs=z(n_pages), free_list=z(n_pages), free_count=z(1),
                      work=z(binding.pages_work_ints(n_rows, n_pages)))
        self.pools = [torch.from_numpy(h).cuda() for h in host]
        self.pt = binding.PageTable(page_size=P, pools=self.pools, **self.t)
        ctx().pages_init(self.pt)
        self.same("init")

    def same(self, what):
        torch.cuda.synchronize()
        g = {n: t.tolist() for n, t in self.t.items()}
        assert g["table"] == self.o.table(), what
        assert g["row_pages"] == [len(r) for r in self.o.rows], what
        assert g["refs"] == self.o.refs(), what
        assert g["free_list"][:g["free_count"][0]] == self.o.free, what
        for a, b in zip(self.pools, self.o.pools):
            assert np.array_equal(a.cpu().numpy(), b), what

    def status(self, n):
        return torch.full((n,), -1, dtype=torch.int32, device="cuda")

    def reserve(self, rows, start, end=None, add=0):
        st = self.status(len(rows))
        ctx().pages_reserve(self.pt, i32(rows), i32(start), i32(end) if end is not None else None, add, st)
        want = self.o.reserve(rows, start, end if end is not None else [s + add for s in start])
        self.same(f"reserve {rows}")
        assert st.tolist() == want

    def fork(self, src, dst):
        st = self.status(len(src))
        ctx().pages_fork(self.pt, i32(src), i32(dst), st)
        want = self.o.fork(src, dst)
        self.same(f"fork {src} {dst}")
        assert st.tolist() == want

    def free(self, rows, keep=None):
        st = self.status(len(rows))
        ctx().pages_free(self.pt, i32(rows), i32(keep) if keep is not None else None, st)
        want = self.o.release(rows, keep if keep is not None else [0] * len(rows))
        self.same(f"free {rows} {keep}")
        assert st.tolist() == want

    def compact(self):
        ctx().pages_compact(self.pt)
        self.o.compact()
        self.same("compact")


def test_a_life():
    b = Both(6, 8, 24, 4)
    b.reserve([0, 1], [0, 0], [10, 5])
    b.fork([0, 0, 1], [2, 3, 4])
    b.reserve([2, 3], [10, 10], add=3)                                    # the page being written copied for both
    b.reserve([1, 4], [4, 4], add=1)                                      # both sharers listed: the last keeps the page
    b.free([0], [5])
    b.compact()
    b.free([2, 0])
    b.compact()
    b.reserve([5, 0], [0, 0], [32, 9])
    b.free([0, 1, 2, 3, 4, 5])
    b.compact()


def test_what_is_refused():
    b = Both(5, 4, 12, 4)
    b.reserve([0, 0, 7, -2, -1, 1, 2, 3], [0, 0, 0, 0, 0, -1, 5, 0], [6, 8, 4, 4, 4, 3, 4, 17])
    b.reserve([4], [0], [0])
    b.fork([0, 0, 0, 9, 0, -1, 1], [1, 1, 0, 2, 9, 3, -1])                # twice, onto itself, outside, passed over
    b.fork([0, 2], [2, 3])                                                # a destination that is a source
    b.fork([0], [1])                                                      # not empty
    b.free([1, 1, 5, -1, 0], [0, 0, 0, 0, -3])
    b.reserve([2, 3, 4], [0, 0, 0], [16, 16, 16])                         # 12 pages needed, fewer there: all or nothing
    b.reserve([2], [0], [16])


def test_a_table_without_pools_and_without_status():
    b = Both(3, 4, 9, 16, n_pools=0)
    ctx().pages_reserve(b.pt, i32([0, 1]), i32([0, 0]), add=33)
    b.o.reserve([0, 1], [0, 0], [33, 33])
    b.same("reserve")
    ctx().pages_free(b.pt, i32([0]))
    b.o.release([0], [0])
    ctx().pages_compact(b.pt)
    b.o.compact()
    b.same("compact")


@pytest.mark.parametrize("seed", range(6))
def test_random_lives(seed):
    rng = random.Random(seed)
    n_rows, max_pages, P = rng.choice([(8, 12, 4), (40, 30, 16), (5, 70, 1)])
    b = Both(n_rows, max_pages, rng.choice([30, 100, 333]), P, n_pools=rng.choice([1, 3]), page_bytes=rng.choice([16, 48, 20000]), seed=seed)
    for _ in range(40):
        rows = [rng.randrange(-1, n_rows) for _ in range(rng.randint(1, n_rows))]
        what = rng.randrange(5)
        if what < 2:
            start = [rng.randrange(0, max_pages * P // 2) for _ in rows]
            if what:
                b.reserve(rows, start, add=rng.randrange(0, 3 * P))
            else:
                b.reserve(rows, start, [s + rng.randrange(0, max_pages * P // 2 + 2) for s in start])
        elif what == 2:
            b.free(rows, [rng.randrange(0, max_pages * P) for _ in rows] if rng.random() < 0.7 else None)
        elif what == 3:
            dst = rng.sample(range(n_rows), min(len(rows), n_rows))
            b.fork(rows[:len(dst)], dst)
        else:
            b.compact()


def test_the_longest_lists_and_a_large_pool():
    n_rows, max_pages, n_pages = 1024, 80, 70001
    b = Both(n_rows, max_pages, n_pages, 8, n_pools=1, page_bytes=16)
    rows = list(range(n_rows))
    random.Random(5).shuffle(rows)
    b.reserve(rows[:512], [0] * 512, [random.Random(i).randrange(1, 640) for i in range(512)])
    b.fork(rows[:512], rows[512:])
    b.reserve(rows, [3] * n_rows, [9] * n_rows)
    b.free(rows[100:1000])
    b.compact()
    b.free(rows)
    assert b.t["free_count"].tolist() == [n_pages]


def test_freed_pages_come_back_in_the_same_order():
    b = Both(4, 16, 40, 4)
    b.reserve([2, 0], [0, 0], [20, 13])
    table = b.t["table"].clone()
    b.free([2, 0])
    b.reserve([2, 0], [0, 0], [20, 13])
    assert torch.equal(table, b.t["table"])


def test_captured_and_replayed():
    b = Both(4, 8, 30, 4)
    b.reserve([0], [0], [10])
    src, dst, start = i32([0, 0]), i32([1, 2]), i32([10, 10])

    def life():
        ctx().pages_free(b.pt, dst)
        ctx().pages_fork(b.pt, src, dst)
        ctx().pages_reserve(b.pt, dst, start, add=4)

    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        life()
    for _ in range(3):
        g.replay()
        b.o.release([1, 2], [0, 0])
        b.o.fork([0, 0], [1, 2])
        b.o.reserve([1, 2], [10, 10], [14, 14])
        b.same("replay")
    del g


@pytest.mark.parametrize("shape", [(16,), (3, 17, 5, 4), (64, 128, 128)])
def test_rows_copied(shape):
    rs = np.random.default_rng(1)
    n = 9
    blocks = [torch.from_numpy(rs.standard_normal((n, *shape)).astype(np.float32)).cuda(), torch.from_numpy(rs.integers(0, 99, (n, 8)).astype(np.int32)).cuda()]
    before = [x.clone() for x in blocks]
    src, dst = [0, 0, 3, -1, 4, 9, 5, 2], [1, 2, 1, 6, -1, 7, 0, 8]
    want = [0, O.SEQ_BAD_ROW, O.SEQ_BAD_ROW, 0, 0, O.SEQ_BAD_ROW, O.SEQ_BAD_ROW, 0]        # 2 and 0 are sources; 1 twice; 9 outside
    st = torch.full((8,), -1, dtype=torch.int32, device="cuda")
    ctx().rows_copy(binding.RowBlocks(blocks), i32(src), i32(dst), st)
    torch.cuda.synchronize()
    assert st.tolist() == want
    for x, y in zip(blocks, before):
        for s, d, w in zip(src, dst, want):
            if s >= 0 and d >= 0 and not w:
                y[d] = y[s].clone()
        assert torch.equal(x, y)

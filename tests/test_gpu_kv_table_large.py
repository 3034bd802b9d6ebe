"""Block tables of hundreds of thousands of rows and millions of pages (skd_kv_assign, skd_kv_compact), against their definition, and in a time
that grows with them and not with their square."""
import ctypes as C

import numpy as np
import pytest
import torch

import kv_scores_reference as S
from paper_2307_02628_amd import skd


def assign(table, pages, page, length, more, source):
    """As kv_scores_reference.assign, in whole arrays."""
    R, W = table.shape
    held = np.clip(length, 0, W * page)
    upto = np.minimum(held + np.maximum(more, 0), W * page)
    start = np.arange(W)[None] * page
    old = np.where(((source >= 0) & (source < R))[:, None], table[np.clip(source, 0, R - 1)], -1)
    rows = np.where((start < upto[:, None]) & (old >= 0) & (old < pages), old, -1)
    write = (upto > held)[:, None] & (start < upto[:, None]) & (start + page > held[:, None])
    named, both = rows >= 0, write & (rows >= 0)
    uses, writes = (np.bincount(rows[m], minlength=pages) for m in (named, both))
    first = np.full(pages, R * W)
    at = np.flatnonzero(both)
    first[rows.ravel()[at][::-1]] = at[::-1]
    here = np.where(named, rows, 0)
    keeps = named & ((uses[here] == 1) | ((uses[here] == writes[here]) & (first[here] == np.arange(R * W).reshape(R, W))))
    wanted = np.flatnonzero(write & ~keeps)
    free = np.flatnonzero(uses == 0)
    missing, copies = max(len(wanted) - len(free), 0), np.zeros((0, 2), np.int64)
    held_there = (start < held[:, None])
    if missing:
        rows = np.where(held_there, rows, -1)
    else:
        flat, free = rows.ravel(), free[:len(wanted)]
        copied = (flat[wanted] >= 0) & held_there.ravel()[wanted]
        copies = np.stack([flat[wanted][copied], free[copied]], 1)
        flat[wanted] = free
    return rows, copies, [len(np.unique(rows[rows >= 0])), missing, len(copies)]


def compact(table, pages):
    there = (table >= 0) & (table < pages)
    used = np.unique(table[there])
    n = len(used)
    far, free = used[used >= n], np.setdiff1d(np.arange(n), used)
    place = np.arange(pages)
    place[far] = free
    return np.where(there, place[np.where(there, table, 0)], -1), np.stack([far, free], 1), [n, 0, len(far)]


def padded(copies, most):
    return np.concatenate([copies, np.full((most - len(copies), 2), -1)])


def random_case(g, R, W, pages, page, forked):
    """Rows with pages of their own up to a length; some forked from others, some with holes and numbers outside of the pool."""
    length = g.integers(0, W * page, R)
    table = np.full((R, W), -1)
    mine = np.arange(W)[None] * page < length[:, None]
    table[mine] = g.permutation(pages)[:mine.sum()]
    table[g.random((R, W)) < 0.01] = -7
    table[g.random((R, W)) < 0.01] = pages
    source = np.where(g.random(R) < forked, g.integers(-1, R + 1, R), np.arange(R))
    length = np.maximum(length[np.clip(source, 0, R - 1)] - g.choice([0, 0, 0, 3], R), 0)
    return table, length, g.choice([0, 1, 1, 1, 40, -2], R), source


def test_the_definitions_agree():
    for seed in range(30):
        g = np.random.default_rng(seed)
        R, W, page = int(g.integers(1, 9)), int(g.integers(1, 5)), 32
        pages = int(g.integers(R * W, 3 * R * W + 2))
        table, length, more, source = random_case(g, R, W, pages, page, 0.5)
        for got, want in ((assign(table.copy(), pages, page, length, more, source), S.assign(table.tolist(), pages, page, length.tolist(), more.tolist(), source.tolist())),
                          (compact(table, pages), S.compact(table.tolist(), pages))):
            assert got[0].tolist() == want[0] and [tuple(c) for c in got[1].tolist()] == want[1] and got[2] == want[2]


class Call:
    """A table on the device, without a pool."""

    def __init__(self, table, pages, page):
        R, W = table.shape
        self.table, self.R, self.pages = self.ints(table), R, pages
        self.kv = skd.Kv(S.BF16, 1, 64, page, pages, R, W, None, self.table.data_ptr())
        lib = skd.lib()
        self.n = max(lib.skd_kv_assign_workspace(C.byref(self.kv)), lib.skd_kv_compact_workspace(C.byref(self.kv)))
        self.ws = torch.randint(-9, 9, (self.n // 4 + 64,), dtype=torch.int32, device="cuda")
        self.ws[self.n // 4:] = 77
        self.out, self.counts = torch.full_like(self.table, 77), torch.full((3,), 77, dtype=torch.int32, device="cuda")

    @staticmethod
    def ints(x):
        return torch.from_numpy(np.ascontiguousarray(x, dtype=np.int32)).cuda()

    def arrays(self, length, more, source):
        self.len, self.more, self.source = (self.ints(x) for x in (length, more, source))
        self.copies = torch.full((self.R, 2), 77, dtype=torch.int32, device="cuda")

    def assign(self):
        assert skd.lib().skd_kv_assign(C.byref(self.kv), self.source.data_ptr(), self.len.data_ptr(), self.more.data_ptr(), self.out.data_ptr(), self.copies.data_ptr(),
                                       self.counts.data_ptr(), self.ws.data_ptr(), self.n, None) == skd.OK

    def compact(self):
        self.copies = torch.full((self.pages // 2, 2), 77, dtype=torch.int32, device="cuda")
        assert skd.lib().skd_kv_compact(C.byref(self.kv), self.out.data_ptr(), self.copies.data_ptr(), self.counts.data_ptr(), self.ws.data_ptr(), self.n, None) == skd.OK

    def check(self, want):
        assert (self.out.cpu().numpy() == want[0]).all() and (self.copies.cpu().numpy() == padded(want[1], len(self.copies))).all() and self.counts.tolist() == want[2]
        assert (self.ws[self.n // 4:] == 77).all()


@pytest.mark.gpu
@pytest.mark.parametrize("R,W,pages", [(1025, 3, 5000), (5000, 2, 1 << 20), (70001, 2, 200000), (1 << 18, 1, 1 << 19), (3, 5, 3 << 20), (2100000, 1, 2500000), (1000, 2, (17 << 20) + 5)])
def test_large_tables(R, W, pages):
    """Around and far beyond a chunk of rows and pages, and a chunk of chunks of either."""
    g = np.random.default_rng(R)
    page = 64
    table, length, more, source = random_case(g, R, W, pages, page, 0.3)
    c = Call(table, pages, page)
    c.arrays(length, more, source)
    c.assign()
    c.check(assign(table.copy(), pages, page, length, more, source))
    c.compact()
    c.check(compact(table, pages))
    c.arrays(length, np.full(R, W * page), source)                   # more than there are, for all but the largest pools
    c.assign()
    c.check(assign(table.copy(), pages, page, length, np.full(R, W * page), source))


@pytest.mark.gpu
def test_time_of_many_rows():
    """2^18 rows of one page: some MB, 0.5 ms.  Sums over all rows in the wave of each row would read 2^37 counts, 30 ms."""
    g = np.random.default_rng(1)
    R, pages = 1 << 18, 1 << 19
    table, length, more, source = random_case(g, R, 1, pages, 32, 0.3)
    c = Call(table, pages, 32)
    c.arrays(length, more, source)
    c.assign()
    begin, end = (torch.cuda.Event(enable_timing=True) for _ in range(2))
    torch.cuda.synchronize()
    begin.record()
    c.assign()
    end.record()
    torch.cuda.synchronize()
    assert begin.elapsed_time(end) < 10.0

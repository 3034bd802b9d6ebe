"""Block tables on the device (skd_kv_assign, skd_kv_compact, skd_kv_copy_pages), against their definition entry by entry, and a
batch that is forked, grown, cut and compacted while it is filed to and attended to."""
import ctypes as C
import math
import random

import pytest
import torch

import kv_scores_reference as S
from paper_2307_02628_amd import skd

pytestmark = pytest.mark.gpu


def ints(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


class Table:
    """A cache of small pages, of which only the table matters."""

    def __init__(self, table, pages, page=32, elem=S.BF16):
        self.table, self.pages, self.page = table, pages, page
        self.pool = torch.randint(0, 255, (pages, 32 // 32 * page // 32 * (4096 * 2 if elem == S.BF16 else 34 * 64)), dtype=torch.uint8, device="cuda",
                                  generator=torch.Generator(device="cuda").manual_seed(1))
        if elem == S.BF16:
            self.pool = self.pool.view(torch.bfloat16)
        self.dev = ints(table).reshape(len(table), -1)
        self.cache = skd.KvCache(self.pool, self.dev, 1, 64, page, elem)

    def assign(self, length, more, source=None, in_place=False, stream=0):
        out = self.dev if in_place else torch.full_like(self.dev, 77)
        copies, counts = torch.full((len(self.table), 2), 77, dtype=torch.int32, device="cuda"), torch.full((3,), 77, dtype=torch.int32, device="cuda")
        ws = torch.randint(-9, 9, (self.cache.assign_workspace() // 4,), dtype=torch.int32, device="cuda")
        self.cache.assign(out, copies, counts, ints(length), ints(more), None if source is None else ints(source), workspace=ws)
        return out.tolist(), copies.tolist(), counts.tolist()

    def compact(self, in_place=False):
        out = self.dev if in_place else torch.full_like(self.dev, 77)
        copies, counts = torch.full((self.pages // 2, 2), 77, dtype=torch.int32, device="cuda"), torch.full((3,), 77, dtype=torch.int32, device="cuda")
        ws = torch.randint(-9, 9, (self.cache.compact_workspace() // 4,), dtype=torch.int32, device="cuda")
        self.cache.compact(out, copies, counts, workspace=ws)
        return out.tolist(), copies.tolist(), counts.tolist()


def padded(result, most):
    rows, copies, counts = result
    return rows, [list(c) for c in copies] + [[-1, -1]] * (most - len(copies)), counts


def random_table(rng, rows, width, pages, named=0.6):
    """Rows that share pages, with holes, numbers outside of the pool, and pages named twice."""
    return [[rng.choice([rng.randrange(pages), rng.randrange(pages), -1, pages, -7]) if rng.random() < named else -1 for _ in range(width)] for _ in range(rows)]


@pytest.mark.parametrize("seed", range(60))
def test_any_table(seed):
    rng = random.Random(seed)
    rows, width = rng.choice([1, 2, 3, 7, 33]), rng.choice([1, 2, 5, 70, 130])
    pages, page = rng.choice([2, 3, 50, 500, 1024, 2500]), rng.choice([32, 64])
    if seed >= 40:                                                   # by the whole chip
        rows, pages = rng.choice([(70, 3000), (130, 300), (7, 5000), (1, 4097), (33, 9000)])
    t = Table(random_table(rng, rows, width, pages, rng.choice([0.1, 0.6, 1.0])), pages, page)
    length = [rng.choice([0, -5, 1, page, rng.randrange(width * page + 1), width * page, 2 ** 31 - 1]) for _ in range(rows)]
    more = [rng.choice([0, 1, 1, -3, page, rng.randrange(4 * page), 2 ** 31 - 1]) for _ in range(rows)]
    source = rng.choice([None, [rng.randrange(-1, rows + 1) for _ in range(rows)], [0] * rows])
    want = padded(S.assign(t.table, pages, page, length, more, source), rows)
    assert t.assign(length, more, source) == want
    if source is None:
        assert t.assign(length, more, in_place=True) == want
    t = Table(t.table, pages, page)
    want = padded(S.compact(t.table, pages), pages // 2)
    assert t.compact() == want
    assert t.compact(in_place=True) == want


def test_a_pool_that_is_full():
    t = Table([[0, 1, -1], [2, -1, -1], [3, -1, -1]], 5)
    for more in ([0, 1, 0], [0, 32, 31], [1, 1, 1], [0, 33, 0], [0, 0, 0], [32, 0, 0]):
        length = [64, 32, 1]
        want = S.assign(t.table, 5, 32, length, more)
        assert t.assign(length, more) == padded(want, 3)
    assert t.assign([64, 32, 1], [1, 1, 1])[2] == [4, 1, 0]          # two were wanted, one was there
    assert t.assign([64, 32, 1], [1, 1, 0])[2] == [4, 1, 0]
    assert t.assign([64, 0, 1], [1, 0, 0])[2] == [4, 0, 0]           # a row ends, its page is dealt out again


def test_many_pages_and_rows():
    rng = random.Random(5)
    rows, width, pages, page = 700, 40, 30000, 32
    order = list(range(pages))
    rng.shuffle(order)
    length = [rng.randrange(1, 30 * page) for _ in range(rows)]
    table = [[order.pop() if i * page < n else -1 for i in range(width)] for n in length]
    t = Table(table, pages, page)
    source, more = [rng.randrange(rows) for _ in range(rows)], [rng.choice([1, 1, 5, 300]) for _ in range(rows)]
    length = [length[s] for s in source]
    assert t.assign(length, more, source) == padded(S.assign(table, pages, page, length, more, source), rows)
    assert t.compact() == padded(S.compact(table, pages), pages // 2)


@pytest.mark.parametrize("pages", [8, 5000])
def test_pages_of_half_a_billion_positions(pages):
    """Places of positions near the end of 32 bits: one page a row, of 2^29 positions, and small rows of many."""
    for page, table in ((1 << 29, [[3], [-1], [3], [0]]), ((1 << 30) // 96, [[1] * 70 + [-1] * 25, [-1] * 95])):
        rows, width = len(table), len(table[0])
        for length, more, source in (([5, 0, 5, 1 << 29], [1, 2, 0, 1], [0, 1, 0, 3]), ([(1 << 30) - 1] * 4, [1 << 29] * 4, [0, 1, 2, 3]), ([1 << 28] * 4, [2 ** 31 - 1] * 4, [0, 0, 0, 0])):
            length, more, source = length[:rows], more[:rows], [min(x, rows - 1) for x in source[:rows]]
            dev, out = ints(table), torch.full((rows, width), 77, dtype=torch.int32, device="cuda")
            kv = skd.Kv(S.BF16, 1, 64, page // 32 * 32, pages, rows, width, None, dev.data_ptr())
            args = [ints(x) for x in (source, length, more)]
            copies, counts = torch.zeros(rows, 2, dtype=torch.int32, device="cuda"), torch.zeros(3, dtype=torch.int32, device="cuda")
            ws = torch.zeros(1 << 18, dtype=torch.uint8, device="cuda")
            rc = skd.lib().skd_kv_assign(C.byref(kv), *[x.data_ptr() for x in args], out.data_ptr(), copies.data_ptr(), counts.data_ptr(), ws.data_ptr(), 1 << 18, None)
            assert rc == skd.OK
            assert (out.tolist(), copies.tolist(), counts.tolist()) == padded(S.assign(table, pages, page // 32 * 32, length, more, source), rows)


def test_a_pool_of_one_page():
    t = Table([[0], [-1]], 1)
    none = torch.zeros(0, 2, dtype=torch.int32, device="cuda")
    out, counts = torch.zeros_like(t.dev), torch.zeros(3, dtype=torch.int32, device="cuda")
    t.cache.compact(out, none, counts, workspace=torch.zeros(t.cache.compact_workspace(), dtype=torch.uint8, device="cuda"))
    assert out.tolist() == [[0], [-1]] and counts.tolist() == [1, 0, 0]
    t.cache.copy_pages(none, counts[2:])


def test_no_rows():
    t = Table([[0, 1]], 4)
    cache = skd.KvCache(t.pool, t.dev[:0], 1, 64, 32, S.BF16)
    counts, none = torch.full((3,), 7, dtype=torch.int32, device="cuda"), torch.zeros(0, dtype=torch.int32, device="cuda")
    ws = torch.zeros(1 << 12, dtype=torch.uint8, device="cuda")
    out, copies = torch.zeros(8, dtype=torch.int32, device="cuda"), torch.full((2, 2), 7, dtype=torch.int32, device="cuda")
    lib = skd.lib()
    assert lib.skd_kv_assign(cache.ref, None, None, None, out.data_ptr(), copies.data_ptr(), counts.data_ptr(), ws.data_ptr(), 1 << 12, None) == skd.OK
    assert counts.tolist() == [0, 0, 0] and (copies == 7).all()
    counts.fill_(7)
    assert lib.skd_kv_compact(cache.ref, out.data_ptr(), copies.data_ptr(), counts.data_ptr(), ws.data_ptr(), 1 << 12, None) == skd.OK
    assert counts.tolist() == [0, 0, 0] and (copies == -1).all()


@pytest.mark.parametrize("elem,page", [(S.BF16, 32), (S.BF16, 96), (S.FP4, 32), (S.FP4, 64)])
def test_copies(elem, page):
    t = Table([[0]], 40, page, elem)
    before = t.pool.clone().view(torch.uint8)
    pairs = [[3, 30], [4, 31], [-1, 5], [6, -1], [40, 7], [8, 40], [9, 9], [2 ** 31 - 1, 10], [3, 33]]
    t.cache.copy_pages(ints(pairs), ints([8]))
    want = before.clone()
    want[30], want[31] = before[3], before[4]
    assert torch.equal(t.pool.view(torch.uint8), want)
    t.cache.copy_pages(ints(pairs), ints([-4]))
    t.cache.copy_pages(ints(pairs), ints([0]))
    t.cache.copy_pages(torch.zeros(0, 2, dtype=torch.int32, device="cuda"))
    assert torch.equal(t.pool.view(torch.uint8), want)
    t.cache.copy_pages(ints(pairs), ints([1000]))                    # no more than there are
    want[33] = before[3]
    assert torch.equal(t.pool.view(torch.uint8), want)


def test_copies_of_large_pages_beyond_32_bits():
    """Pages of an odd number of pieces, behind 4 GiB."""
    H, page = 3, 160
    size = H * page * (2 * 128 + 2)
    pages = (5 << 30) // size
    pool = torch.zeros(pages, size, dtype=torch.uint8, device="cuda")
    pool[pages - 1] = torch.randint(0, 255, (size,), dtype=torch.uint8, device="cuda")
    pool[1] = torch.randint(0, 255, (size,), dtype=torch.uint8, device="cuda")
    cache = skd.KvCache(pool, ints([[0]]), H, 128, page, S.FP8)
    cache.copy_pages(ints([[pages - 1, 0], [1, pages - 2]]))
    assert torch.equal(pool[0], pool[pages - 1]) and torch.equal(pool[pages - 2], pool[1]) and not pool[2].any() and not pool[pages - 3].any()


@pytest.mark.parametrize("elem", [S.BF16, S.FP8, S.FP4])
def test_a_batch_that_is_forked_cut_and_compacted(elem):
    """Beams over one prompt: they go on from each other, take drafts back, end, grow into new pages and are moved, and what each
    row attends to stays what it was."""
    H, dh, page, beams, pages, width = 2, 64, 32, 4, 40, 6
    g = torch.Generator().manual_seed(3)
    pool = S.garbage(elem, pages, H, dh, page)
    copies, counts = torch.zeros(pages // 2, 2, dtype=torch.int32, device="cuda"), torch.zeros(3, dtype=torch.int32, device="cuda")
    few = torch.zeros(beams, 2, dtype=torch.int32, device="cuda")
    tables = [torch.full((beams, width), -1, dtype=torch.int32, device="cuda") for _ in range(2)]
    caches = [skd.KvCache(pool, t, H, dh, page, elem) for t in tables]
    ws = torch.zeros(max(caches[0].assign_workspace(), caches[0].compact_workspace()), dtype=torch.uint8, device="cuda")
    rows, now = [([], []) for _ in range(beams)], 0                  # keys and values of each beam, on the host
    rng = random.Random(7)
    for step in range(24):
        if step == 0:
            source, length, more = [0, -1, -1, -1], [0, 0, 0, 0], [45, 0, 0, 0]
        elif step == 1:
            source, length, more = [0, 0, 0, 0], [45] * 4, [1] * 4
        else:
            source = [rng.choice([b, rng.randrange(beams)]) for b in range(beams)]
            length = [max(len(rows[s][0]) - rng.choice([0, 0, 3]), 40) for s in source]
            more = [rng.choice([1, 1, 2, 9, 0]) for _ in range(beams)]
        caches[now].assign(tables[1 - now], few, counts, ints(length), ints(more), ints(source), workspace=ws)
        now = 1 - now
        caches[now].copy_pages(few, counts[2:])
        if step % 5 == 4:
            caches[now].compact(tables[now], copies, counts, workspace=ws)
            caches[now].copy_pages(copies, counts[2:])
            pages_now = {p for row in tables[now].tolist() for p in row if p >= 0}
            assert pages_now == set(range(counts[0].item()))
        assert counts[1].item() == 0
        rows = [(list(rows[s][0][:n]), list(rows[s][1][:n])) if s >= 0 else ([], []) for s, n in zip(source, length)]
        k, v = (torch.randn(sum(more), H, dh, generator=g).bfloat16() for _ in range(2))
        q = torch.randn(sum(more), 2 * H, dh, generator=g).bfloat16().cuda()
        at = 0
        for b, n in enumerate(more):
            rows[b][0].extend(k[at:at + n])
            rows[b][1].extend(v[at:at + n])
            at += n
        if not sum(more):
            continue
        first = ints([0] + torch.tensor(more).cumsum(0).tolist())
        ch = skd.KvChunk(first, ints(length), sum(more), max(more), max(length))
        out, sc = torch.zeros_like(q), skd.KvScores(cap=8.0, window=64)
        space = torch.empty(caches[now].attend_scores_workspace(ch, 2 * H, sc), dtype=torch.uint8, device="cuda")
        caches[now].attend_scores(ch, q, out, 1 / math.sqrt(dh), sc, k.cuda(), v.cuda(), workspace=space)
        at = 0
        for b, n in enumerate(more):
            if n:
                kh, vh = (torch.from_numpy(S.as_held(torch.stack(x).double().numpy(), elem)) for x in rows[b])
                ref, bound = S.attention(q[at:at + n].cpu().double(), kh, vh, length[b], 1 / math.sqrt(dh), cap=8.0, window=64)
                assert ((out[at:at + n].cpu().double() - ref).abs() <= bound).all(), (step, b)
            at += n


def test_captured_and_replayed():
    rng = random.Random(9)
    rows, width, pages = 6, 5, 60
    t = Table(random_table(rng, rows, width, pages), pages)
    dev = {n: torch.zeros(rows, dtype=torch.int32, device="cuda") for n in ("len", "more", "source")}
    out, copies, counts = torch.zeros_like(t.dev), torch.zeros(rows, 2, dtype=torch.int32, device="cuda"), torch.zeros(3, dtype=torch.int32, device="cuda")
    out2, moves, counts2 = torch.zeros_like(t.dev), torch.zeros(pages // 2, 2, dtype=torch.int32, device="cuda"), torch.zeros(3, dtype=torch.int32, device="cuda")
    ws = torch.zeros(max(t.cache.assign_workspace(), t.cache.compact_workspace()), dtype=torch.uint8, device="cuda")
    then = skd.KvCache(t.pool, out, 1, 64, 32)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        s = torch.cuda.current_stream().cuda_stream
        t.cache.assign(out, copies, counts, dev["len"], dev["more"], dev["source"], workspace=ws, stream=s)
        t.cache.copy_pages(copies, counts[2:], stream=s)
        then.compact(out2, moves, counts2, workspace=ws, stream=s)
        then.copy_pages(moves, counts2[2:], stream=s)
    for _ in range(5):
        table = random_table(rng, rows, width, pages)
        length, more, source = [rng.randrange(100) for _ in range(rows)], [rng.randrange(40) for _ in range(rows)], [rng.randrange(rows) for _ in range(rows)]
        t.dev.copy_(ints(table))
        for n, x in (("len", length), ("more", more), ("source", source)):
            dev[n].copy_(ints(x))
        before = t.pool.clone()
        g.replay()
        torch.cuda.synchronize()
        first = S.assign(table, pages, 32, length, more, source)
        second = S.compact(first[0], pages)
        assert (out.tolist(), copies.tolist(), counts.tolist()) == padded(first, rows)
        assert (out2.tolist(), moves.tolist(), counts2.tolist()) == padded(second, pages // 2)
        for a, b in first[1] + second[1]:
            before[b] = before[a]
        assert torch.equal(t.pool.view(torch.uint8), before.view(torch.uint8))


def test_refusals_of_memory():
    t = Table([[0, 1], [2, -1]], 4)
    ws = torch.zeros(t.cache.assign_workspace() + t.cache.compact_workspace(), dtype=torch.uint8, device="cuda")
    dev = torch.zeros(64, dtype=torch.int32, device="cuda")
    host = torch.zeros(64, dtype=torch.int32)
    lib, n = skd.lib(), ws.numel()

    def assign(source=None, length=dev, more=dev, out=dev[8:], copies=dev[16:], counts=dev[32:], space=ws, n=n):
        return lib.skd_kv_assign(t.cache.ref, None if source is None else source.data_ptr(), length.data_ptr(), more.data_ptr(), out.data_ptr(), copies.data_ptr(),
                                 counts.data_ptr(), space.data_ptr(), n, None)

    assert assign() == skd.OK
    assert assign(length=host) == assign(more=host) == assign(out=host) == assign(copies=host) == assign(counts=host) == assign(source=host) == skd.ERR_RANGE
    assert assign(space=torch.zeros(n, dtype=torch.uint8)) == skd.ERR_RANGE
    assert assign(n=t.cache.assign_workspace() - 1) == skd.ERR_NOMEM
    assert assign(out=t.dev) == skd.OK and assign(source=dev, out=t.dev) == skd.ERR_RANGE
    assert assign(out=t.dev.view(-1)[1:]) == skd.ERR_RANGE
    assert lib.skd_kv_copy_pages(t.cache.ref, host.data_ptr(), 1, None, None) == lib.skd_kv_copy_pages(t.cache.ref, dev.data_ptr(), 1, host.data_ptr(), None) == skd.ERR_RANGE
    with pytest.raises(ValueError):
        t.cache.assign(dev, dev.view(-1, 2), dev[:3], dev[:2], dev[:2], workspace=ws)
    with pytest.raises(ValueError):
        t.cache.copy_pages(dev[:3].view(1, 3))

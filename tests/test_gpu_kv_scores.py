"""Attention with capped scores, scores that fall with the distance, windows, documents and prefixes (skd_kv_attend_scores), against 64
bits on the CPU."""
import math

import numpy as np
import pytest
import torch

import kv_scores_reference as S
from paper_2307_02628_amd import skd

pytestmark = pytest.mark.gpu
ELEMS = [S.BF16, S.FP8, S.FP4]


def queries(tokens, heads, dh, size=1.0, seed=1):
    return (size * torch.randn(tokens, heads, dh, generator=torch.Generator().manual_seed(seed))).bfloat16().cuda()


def documents(past, new, mean, seed=0):
    """begin of each token: rows are cut at random places."""
    g, begin = np.random.default_rng(seed), []
    for p, n in zip(past, new):
        first = np.maximum.accumulate(np.where(g.random(p + n) < 1 / mean, np.arange(p + n), 0))
        begin += first[p:].tolist()
    return begin


def positions(past, new):
    return [p + i for p, n in zip(past, new) for i in range(n)]


SHAPES = [
    # H, group, dh, page, past, new
    (4, 1, 64, 64, [31, 20], [1, 1]),
    (2, 1, 128, 64, [0, 64, 33, 700], [1, 1, 1, 1]),
    (3, 4, 128, 32, [100, 0, 1500], [1, 1, 1]),
    (1, 8, 64, 96, [5, 40], [3, 2]),
    (2, 3, 128, 64, [0, 63, 17], [5, 7, 0]),
    (2, 20, 64, 64, [70, 2], [1, 1]),
    (2, 1, 128, 64, [0, 300, 9], [70, 33, 1]),
    (1, 2, 64, 128, [130, 0], [129, 64]),
    (2, 2, 128, 64, [1000, 31], [200, 257]),
]
CHANGES = ["cap", "slopes", "window", "documents", "prefix", "all"]


def change(name, heads, past, new):
    slopes = [2.0 ** (-8 * (h + 1) / heads) for h in range(heads)]
    if name == "cap":
        return dict(cap=5.0)
    if name == "slopes":
        return dict(slopes=slopes)
    if name == "window":
        return dict(window=37)
    if name == "documents":
        return dict(begin=documents(past, new, 40))
    if name == "prefix":
        return dict(end=[max(p + 1, 150 if p < 150 else 0) for p in positions(past, new)])
    return dict(cap=20.0, slopes=slopes, window=300, begin=documents(past, new, 200), end=[p + 1 + p % 50 for p in positions(past, new)])


@pytest.mark.parametrize("name", CHANGES)
@pytest.mark.parametrize("elem", ELEMS)
@pytest.mark.parametrize("H,group,dh,page,past,new", SHAPES)
def test_attention(H, group, dh, page, past, new, elem, name):
    c = S.Rows(elem, H, dh, page, past, new, seed=11 + group, spare=1)
    q = queries(sum(new), H * group, dh, 3.0)
    if max(past):
        c.append([0] * len(past), past)
    how = change(name, H * group, past, new)
    out = c.attend(q, files=True, **how)
    c.check(q, out, **how)
    again = c.attend(q, **how)                                       # the cache holds the tokens now
    c.check(q, again, **how)
    assert torch.equal(again, out) or max(new) == 1
    assert torch.equal(again, c.attend(q, **how))
    k, v = c.read([0] * len(past), c.total)
    assert torch.equal(k.double(), c.held(c.k, [0] * len(past), c.total)) and torch.equal(v.double(), c.held(c.v, [0] * len(past), c.total))


@pytest.mark.parametrize("elem", ELEMS)
@pytest.mark.parametrize("new", [1, 9, 140])
def test_nothing_changed_is_the_attention_itself(elem, new):
    c = S.Rows(elem, 2, 128, 64, [500, 3], [new, new], seed=3)
    c.append([0, 0], c.total)
    q = queries(2 * new, 4, 128)
    out = c.attend(q, cap=0.0, end=[p + 1 for p in positions(c.past, c.new)])
    c.check(q, out)
    plain = c.attend(q)
    c.check(q, plain)
    wide = c.attend(q, window=1 << 31 - 1, begin=[-5] * (2 * new))
    assert torch.equal(wide, out)


@pytest.mark.parametrize("cap", [2.0 ** -20, 0.5, 50.0, 1024.0])
@pytest.mark.parametrize("new", [1, 40, 130])
def test_caps(cap, new):
    """From caps that leave hardly any difference of scores to those that hardly bend them."""
    c = S.Rows(S.BF16, 2, 64, 64, [200], [new], seed=7)
    c.append([0], c.total)
    q = queries(new, 2, 64, 10.0)
    c.check(q, c.attend(q, cap=cap), cap=cap)


@pytest.mark.parametrize("elem", ELEMS)
@pytest.mark.parametrize("slope", [0.0, -0.05, 30.0])
@pytest.mark.parametrize("new", [1, 5, 150])
def test_slopes(elem, slope, new):
    """No share, one that grows with the distance, one that leaves the nearest position alone."""
    c = S.Rows(elem, 2, 64, 32, [300, 40], [new, new], seed=9)
    c.append([0, 0], c.total)
    q = queries(2 * new, 4, 64)
    how = dict(slopes=[slope, 0.0, slope / 7, 1.0])
    c.check(q, c.attend(q, **how), **how)
    how["end"] = [c.past[i // new] + new for i in range(2 * new)]    # in both directions
    c.check(q, c.attend(q, **how), **how)


@pytest.mark.parametrize("elem", ELEMS)
@pytest.mark.parametrize("new,group", [(1, 1), (1, 4), (3, 2), (20, 2), (140, 1), (300, 2)])
def test_tokens_that_see_nothing(elem, new, group):
    """Empty ranges among others, of all tokens, and bounds far outside of what there is."""
    c = S.Rows(elem, 2, 64, 64, [70, 0], [new, new], seed=13)
    c.append([0, 0], c.past) if max(c.past) else None
    q = queries(2 * new, 2 * group, 64)
    at = positions(c.past, c.new)
    cases = [dict(begin=[p + 1 if i % 3 == 0 else 0 for i, p in enumerate(at)]),
             dict(end=[0 if i % 2 else p + 1 for i, p in enumerate(at)]),
             dict(begin=[2 ** 31 - 1] * len(at)), dict(end=[-2 ** 31] * len(at)), dict(end=[2 ** 31 - 1] * len(at), begin=[-2 ** 31] * len(at)),
             dict(begin=[64] * len(at), end=[96] * len(at)),                       # one whole block and nothing else
             dict(begin=at), dict(window=1), dict(window=2 ** 31 - 1, cap=3.0)]
    for how in cases:
        out = c.attend(q, files=True, **how)
        c.check(q, out, **how)
        lo, hi = zip(*(S.ranges(p, n, how.get("window", 0), *(None if how.get(x) is None else np.array(how[x][r * new:(r + 1) * new]) for x in ("begin", "end")))
                       for r, (p, n) in enumerate(zip(c.past, c.new))))
        empty = torch.from_numpy(np.concatenate(lo) >= np.concatenate(hi))
        assert (out[empty] == 0).all()


@pytest.mark.parametrize("elem", ELEMS)
@pytest.mark.parametrize("new", [1, 4, 70, 200])
def test_infinities_outside_of_what_a_query_sees(elem, new):
    """What is not finite before or behind a token's positions does not reach it; what it sees does."""
    past = [100, 10]
    c = S.Rows(elem, 2, 64, 64, past, [new, new], seed=31)
    c.v[0][30, 0, 3], c.v[0][31, 1, 40], c.v[0][99, 0, 33] = float("inf"), float("nan"), float("-inf")
    c.k[0][5, 0, 0], c.k[0][90, 1, 7] = float("nan"), float("inf")
    c.v[1][10 + new - 1, 1, 5] = float("-inf")
    c.append([0, 0], c.total)
    q = queries(2 * new, 4, 64)
    begin = [(32 if i % 2 else 6) if i < new else 0 for i in range(2 * new)]
    begin = [100 if i % 5 == 4 and i < new else b for i, b in enumerate(begin)]
    for how in (dict(begin=begin), dict(begin=begin, cap=10.0), dict(window=40)):
        out = c.attend(q, **how).double()
        for r in range(2):
            k, v = (torch.from_numpy(S.as_held(x[r].double().numpy(), elem)) for x in (c.k, c.v))
            lo, hi = S.ranges(past[r], new, how.get("window", 0), np.array(begin[r * new:(r + 1) * new]) if "begin" in how else None)
            for i in range(new):
                for h in range(4):
                    me = slice(int(lo[i]), int(hi[i]))
                    s = q[r * new + i, h].cpu().double() @ k[me, h // 2].t() / 8
                    s = 10 * torch.tanh(s / 10) if "cap" in how else s
                    w = torch.softmax(s, -1)
                    ref, got = (w[:, None] * v[me, h // 2]).sum(0), out[r * new + i, h]
                    where = (how.keys(), r, i, h)
                    assert torch.equal(torch.isnan(got), torch.isnan(ref)), where
                    assert torch.equal(got.isposinf(), ref.isposinf()) and torch.equal(got.isneginf(), ref.isneginf()), where
                    ok = torch.isfinite(ref)
                    assert ((got - ref)[ok].abs() <= 2.0 ** -7 * 8).all(), where  # (the bound of the reference, coarser: |v| is below 8)


@pytest.mark.parametrize("elem", ELEMS)
def test_rows_without_pages_holes_and_rows_behind_the_last(elem):
    c = S.Rows(elem, 2, 64, 32, [40, 20], [2, 3], seed=41)
    c.append([0, 0], c.total)
    q = queries(8, 2, 64)
    ch = skd.KvChunk(torch.tensor([0, 2, 5], dtype=torch.int32, device="cuda"), torch.tensor([40, 20], dtype=torch.int32, device="cuda"), 8, 3, 40)
    sc = c.scores(2, cap=4.0, begin=[0] * 8)
    ws = torch.empty(c.cache.attend_scores_workspace(ch, 2, sc), dtype=torch.uint8, device="cuda")
    out = torch.full_like(q, 3.0)
    c.cache.attend_scores(ch, q, out, 0.125, sc, workspace=ws)
    c.check(q[:5], out[:5].cpu(), cap=4.0)
    assert (out[5:] == 3).all()
    none = skd.KvCache(c.pool, torch.full_like(c.table, -1).cuda(), 2, 64, 32, elem)
    none.attend_scores(ch, q, out, 0.125, sc, workspace=ws)
    assert (out[:5] == 0).all() and (out[5:] == 3).all()
    # a token whose page is none: dropped, and nobody sees it
    lost = c.table.clone()
    lost[0, 1] = -1
    torch.cuda.synchronize()
    one = skd.KvChunk(torch.tensor([0, 1, 1], dtype=torch.int32, device="cuda"), torch.tensor([40, 0], dtype=torch.int32, device="cuda"), 1, 1, 40)
    cache = skd.KvCache(c.pool, lost.cuda(), 2, 64, 32, elem)
    sc = c.scores(2, window=9)                                       # positions 32 .. 40, all on the lost page
    k, v = (torch.ones(1, 2, 64, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    cache.attend_scores(one, q[:1], out[:1], 0.125, sc, k, v, workspace=ws)
    assert (out[:1] == 0).all()
    with pytest.raises(ValueError):
        c.cache.attend_scores(ch, q, out, 0.125, c.scores(2, begin=[0] * 5), workspace=ws)
    with pytest.raises(ValueError):
        c.cache.attend_scores(ch, q, out, 0.125, c.scores(2, slopes=[1.0]), workspace=ws)
    host = skd.KvScores(end=torch.zeros(8, dtype=torch.int32))
    with pytest.raises(skd.SkdError) as e:
        c.cache.attend_scores(ch, q, out, 0.125, host, workspace=ws)
    assert e.value.code == skd.ERR_RANGE


@pytest.mark.parametrize("elem", ELEMS)
@pytest.mark.parametrize("new", [1, 6, 90])
def test_strided_queries_keys_values_and_outputs(elem, new):
    """All of them columns of wider rows, as a projection leaves them; what lies between stays."""
    c = S.Rows(elem, 2, 64, 64, [70, 31], [new, new], seed=19)
    c.append([0, 0], c.past)
    T, W = 2 * new, 2 * 64
    packed = torch.full((T, 4 * W + 8), 9.0, dtype=torch.bfloat16, device="cuda")
    q, k, v = packed[:, :2 * W], packed[:, 2 * W:3 * W], packed[:, 3 * W:4 * W]
    q.copy_(queries(T, 4, 64).flatten(1))
    k.copy_(c.tokens(c.k, c.past, c.new).flatten(1))
    v.copy_(c.tokens(c.v, c.past, c.new).flatten(1))
    wide = torch.full((T, 3 * W), 7.0, dtype=torch.bfloat16, device="cuda")
    ch, how = c.chunk(c.past, c.new), dict(cap=9.0, slopes=[0.1, 0.0, 1.0, 0.02], window=50)
    sc = c.scores(4, **how)
    ws = torch.empty(c.cache.attend_scores_workspace(ch, 4, sc), dtype=torch.uint8, device="cuda")
    c.cache.attend_scores(ch, q, wide[:, 8:8 + 2 * W], 0.125, sc, k, v, workspace=ws)
    c.check(q.unflatten(1, (4, 64)), wide[:, 8:8 + 2 * W].unflatten(1, (4, 64)).cpu(), 0.125, **how)
    assert (wide[:, :8] == 7).all() and (wide[:, 8 + 2 * W:] == 7).all() and (packed[:, 4 * W:] == 9).all()
    kr, vr = c.read([0, 0], c.total)
    assert torch.equal(kr.double(), c.held(c.k, [0, 0], c.total)) and torch.equal(vr.double(), c.held(c.v, [0, 0], c.total))


def test_two_streams_at_once():
    """Other rows, masks and workspaces on two streams at a time, over one pool, against the same calls one after the other."""
    c = S.Rows(S.FP4, 4, 128, 64, [3000, 2500], [1, 1], seed=29)
    c.append([0, 0], c.total)
    q = queries(2, 16, 128)
    sc = [c.scores(16, slopes=[0.01 * h for h in range(16)]), c.scores(16, cap=20.0, window=1000)]
    ch = c.chunk(c.past, c.new)
    spaces = [torch.empty(c.cache.attend_scores_workspace(ch, 16, x), dtype=torch.uint8, device="cuda") for x in sc]
    want = [torch.zeros_like(q) for _ in sc]
    for i in range(2):
        c.cache.attend_scores(ch, q, want[i], 0.1, sc[i], workspace=spaces[i])
    outs, streams = [torch.zeros_like(q) for _ in sc], [torch.cuda.Stream() for _ in sc]
    torch.cuda.synchronize()
    for _ in range(20):
        for i in range(2):
            c.cache.attend_scores(ch, q, outs[i], 0.1, sc[i], workspace=spaces[i], stream=streams[i].cuda_stream)
    torch.cuda.synchronize()
    assert torch.equal(outs[0], want[0]) and torch.equal(outs[1], want[1])
    c.check(q, outs[1].cpu(), 0.1, cap=20.0, window=1000)


def test_many_rows_of_all_lengths():
    """More rows than compute units, from none to some hundreds of positions, each with a prefix of its own."""
    g = np.random.default_rng(5)
    past, new = g.integers(0, 300, 150).tolist(), g.integers(0, 9, 150).tolist()
    new[3], past[3] = 0, 0
    c = S.Rows(S.BF16, 1, 64, 32, past, new, seed=37)
    c.append([0] * 150, past)
    q = queries(sum(new), 3, 64)
    end = [max(p + 1, int(w)) for p, w in zip(positions(past, new), g.integers(0, 400, sum(new)))]
    out = c.attend(q, files=True, end=end, slopes=[0.5, 0.05, 0.0])
    c.check(q, out, end=end, slopes=[0.5, 0.05, 0.0])


@pytest.mark.parametrize("elem", ELEMS)
def test_long_rows_in_shares(elem):
    """Shares of the keys joined: windows that end inside shares, distances of a long row."""
    c = S.Rows(elem, 1, 128, 64, [9000], [2], seed=43)
    c.append([0], c.total)
    q = queries(2, 4, 128)
    for how in (dict(slopes=[0.5, 0.01, 0.0, 1e-4]), dict(window=4097), dict(begin=[8999, 0], cap=30.0), dict(begin=[4500, 8990], end=[4532, 9000])):
        c.check(q, c.attend(q, **how), **how)


def test_captured_and_replayed():
    """A step and a chunk with slopes, windows and documents, captured once and replayed with other tokens, lengths and documents, on a
    stream of its own, against the same calls made directly."""
    for elem, new in ((S.BF16, 1), (S.FP4, 1), (S.FP8, 40), (S.FP4, 40)):
        c = S.Rows(elem, 2, 128, 64, [900, 31], [new, new], seed=51, spare=1)
        c.append([0, 0], c.total)
        first = torch.tensor([0, new, 2 * new], dtype=torch.int32, device="cuda")
        past = torch.tensor(c.past, dtype=torch.int32, device="cuda")
        ch = skd.KvChunk(first, past, 2 * new, new, 1000)
        q, k, v = (torch.zeros(2 * new, n, 128, dtype=torch.bfloat16, device="cuda") for n in (4, 2, 2))
        sc = c.scores(4, cap=20.0, slopes=[0.5, 0.1, 0.0, 0.01], window=300, begin=[0] * 2 * new)
        begin = sc._keep[1]
        outs, graphs = [torch.zeros_like(q) for _ in range(2)], []
        spaces = [torch.empty(c.cache.attend_scores_workspace(ch, 4, sc), dtype=torch.uint8, device="cuda") for _ in range(3)]
        for i in range(2):
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g):
                c.cache.attend_scores(ch, q, outs[i], 0.1, sc, k, v, workspace=spaces[i], stream=torch.cuda.current_stream().cuda_stream)
            graphs.append(g)
        gen = torch.Generator(device="cuda").manual_seed(9)
        for step in range(3):
            for t in (q, k, v):
                t.copy_(torch.randn(t.shape, generator=gen, device="cuda"))
            past.copy_(torch.tensor([900 - 100 * step, 31 + step - (new > 1) * 5], dtype=torch.int32))
            begin.copy_(torch.randint(0, 100, begin.shape, generator=gen, device="cuda"))
            want = torch.zeros_like(q)
            c.cache.attend_scores(ch, q, want, 0.1, sc, k, v, workspace=spaces[2])
            torch.cuda.synchronize()
            pool = c.pool.clone()
            for g in graphs:
                g.replay()
            torch.cuda.synchronize()
            assert torch.equal(outs[0], want) and torch.equal(outs[1], want)
            assert torch.equal(c.pool.view(torch.uint8), pool.view(torch.uint8))

"""The operators on a paged cache and the draw as a server uses them: prompts in pieces, then a token a row and step (filed, attended
to, drawn from, the next row of the cache), drafts that are taken back; and long rows of many pages."""
import math

import numpy as np
import pytest
import torch

import kv_reference as R
from paper_2307_02628_amd import skd
from test_gpu_kv_ops import Case
from test_gpu_sample_rows import reference

pytestmark = pytest.mark.gpu


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


class Model:
    """One layer of attention: keys, values and queries of a token by lookup, logits by a product that is exact in fp32 up to its
    own sums (the draw is checked against the logits themselves)."""

    def __init__(self, H, group, dh, V, seed):
        g = torch.Generator().manual_seed(seed)
        self.q, self.k, self.v = (torch.randn(V, n, dh, generator=g).bfloat16().cuda() for n in (H * group, H, H))
        self.out = (torch.randn(H * group * dh, V, generator=g) * 0.3).cuda()
        self.H, self.group, self.dh, self.V = H, group, dh, V

    def logits(self, o):
        return o.float().flatten(1) @ self.out


class Server:
    def __init__(self, m, elem, lens, room, page, seed):
        self.m, self.elem, B = m, elem, len(lens)
        need = -(-room // page)
        self.table = torch.randperm(B * need, generator=torch.Generator().manual_seed(seed)).view(B, need).int().cuda()
        size = skd.KvCache(torch.empty(1, m.H * page * 2 * m.dh, dtype=torch.bfloat16, device="cuda"), self.table, m.H, m.dh, page).page_bytes
        size = size // 2 + m.H * page * 2 if elem == R.FP8 else size
        self.pool = torch.full((B * need, size), 0xff, dtype=torch.uint8, device="cuda")
        self.cache = skd.KvCache(self.pool, self.table, m.H, m.dh, page, elem)
        self.past, self.first = i32(lens) * 0, torch.arange(B + 1, dtype=torch.int32, device="cuda")
        self.step_ = skd.KvChunk(self.first, self.past, B, 1, room)
        self.ws = torch.empty(self.cache.attend_workspace(self.step_, m.H * m.group), dtype=torch.uint8, device="cuda")
        self.draw_ws = torch.empty(skd.sample_workspace(B, m.V), dtype=torch.uint8, device="cuda")
        self.tok, self.logits = torch.zeros(B, dtype=torch.int32, device="cuda"), torch.zeros(B, m.V, device="cuda")
        self.o = torch.zeros(B, m.H * m.group, m.dh, dtype=torch.bfloat16, device="cuda")

    def pieces(self, tokens, counts):
        """`counts` next tokens of each row at once; the last output of each."""
        m, t = self.m, torch.cat(tokens).cuda()
        ch = skd.KvChunk(i32([0] + list(np.cumsum(counts))), self.past, len(t), max(counts), 1 << 20)
        o = torch.empty_like(m.q[t])
        ws = torch.empty(self.cache.attend_workspace(ch, m.H * m.group), dtype=torch.uint8, device="cuda")
        self.cache.attend(ch, m.q[t], o, 1 / math.sqrt(m.dh), m.k[t], m.v[t], workspace=ws)
        self.past += i32(counts)
        return o

    def step(self, u, params, stream=0):
        """The tokens in self.tok are filed and attended to; the next ones are drawn into it."""
        m, t = self.m, self.tok.long()
        self.cache.attend(self.step_, m.q[t], self.o, 1 / math.sqrt(m.dh), m.k[t], m.v[t], workspace=self.ws, stream=stream)
        self.logits.copy_(m.logits(self.o))
        skd.sample(self.logits, u, self.tok, *params, workspace=self.draw_ws, stream=stream)
        self.past += 1

    def check(self, history, o):
        """o [rows][heads][dh]: outputs of the last token of each row's history."""
        m = self.m
        for r, h in enumerate(history):
            t = torch.tensor(h)
            k, v = (torch.from_numpy(R.as_held(x.cpu()[t].double().numpy(), self.elem)) for x in (m.k, m.v))
            ref, bound = R.attention(m.q.cpu()[t[-1:]].double(), k, v, len(h) - 1, 1 / math.sqrt(m.dh))
            assert ((o[r].cpu().double() - ref[0]).abs() <= bound[0]).all(), r


@pytest.mark.parametrize("elem", [R.BF16, R.FP8])
@pytest.mark.parametrize("H,group,dh,page", [(2, 1, 64, 32), (2, 4, 128, 64)])
def test_prompts_in_pieces_then_steps(elem, H, group, dh, page):
    V, lens, B = 701, [45, 130, 1, 77], 4
    m = Model(H, group, dh, V, 5)
    g = torch.Generator().manual_seed(6)
    prompts = [torch.randint(0, V, (n,), generator=g) for n in lens]
    params = (torch.tensor([0.7, 1.0, 0.0, 1.3]).cuda(), i32([0, 40, 0, 5]), torch.tensor([0.9, 1.0, 1.0, 0.8]).cuda(), torch.tensor([0.0, 0.02, 0.0, 0.0]).cuda())
    us = torch.rand(8, B, generator=g).cuda()
    u = torch.zeros(B, device="cuda")

    def prefilled(cuts):
        s = Server(m, elem, lens, 160, page, 7)
        for a, b in zip(cuts, cuts[1:]):
            part = [p[min(a, len(p)):min(b, len(p))] for p in prompts]
            s.pieces(part, [len(p) for p in part])
        s.tok.copy_(i32([p[0] for p in prompts]))
        assert s.past.tolist() == lens
        return s

    eager, captured = prefilled([0, 130]), prefilled([0, 3, 68, 100, 130])
    # the same tokens in other pieces: the same pages (a row's own, dealt out alike)
    k, v = (torch.empty(2, sum(lens), H, dh, device="cuda") for _ in range(2))
    whole = skd.KvChunk(i32([0] + list(np.cumsum(lens))), i32([0] * B), sum(lens), max(lens), 0)
    for i, s in enumerate((eager, captured)):
        s.cache.read(whole, k[i], v[i])
    assert torch.equal(k[0], k[1]) and torch.equal(v[0], v[1])
    torch.cuda.synchronize()
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    start = captured.past.clone(), captured.tok.clone()
    with torch.cuda.stream(side):
        captured.step(u, params, side.cuda_stream)                     # (libraries choose and allocate before a capture)
    side.synchronize()
    with torch.cuda.graph(graph):
        captured.step(u, params, torch.cuda.current_stream().cuda_stream)
    captured.past.copy_(start[0])
    captured.tok.copy_(start[1])
    history = [p.tolist() for p in prompts]
    for i in range(8):
        for h, t in zip(history, eager.tok.tolist()):
            h.append(t)
        u.copy_(us[i])
        eager.step(u, params)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(eager.o, captured.o) and torch.equal(eager.tok, captured.tok) and torch.equal(eager.past, captured.past)
        eager.check(history, eager.o)
        z, col = eager.logits.cpu().numpy(), [p.cpu().numpy() for p in params]
        want = [reference(z[b], float(us[i, b]), float(col[0][b]), int(col[1][b]), float(col[2][b]), float(col[3][b])) for b in range(B)]
        assert eager.tok.tolist() == want


@pytest.mark.parametrize("elem", [R.BF16, R.FP8])
def test_drafts_that_are_taken_back(elem):
    """Five drafted tokens a row at once give what five steps give within rounding; the rows then go on from different places."""
    V, B = 300, 3
    m = Model(2, 2, 64, V, 8)
    g = torch.Generator().manual_seed(9)
    prompts = [torch.randint(0, V, (n,), generator=g) for n in (60, 33, 2)]
    drafts = [torch.randint(0, V, (5,), generator=g) for _ in range(B)]
    s = Server(m, elem, [60, 33, 2], 96, 32, 10)
    s.pieces(prompts, [60, 33, 2])
    o = s.pieces(drafts, [5] * B).view(B, 5, 4, 64)
    history = [p.tolist() for p in prompts]
    for i in range(5):
        s.check([h + d[:i + 1].tolist() for h, d in zip(history, drafts)], o[:, i])
    taken = [0, 5, 2]
    s.past.copy_(i32([len(h) + n for h, n in zip(history, taken)]))
    history = [h + d[:n].tolist() for h, d, n in zip(history, drafts, taken)]
    more = [torch.randint(0, V, (3,), generator=g) for _ in range(B)]
    o = s.pieces(more, [3] * B).view(B, 3, 4, 64)
    s.check([h + x.tolist() for h, x in zip(history, more)], o[:, 2])


@pytest.mark.parametrize("elem", [R.BF16, R.FP8])
@pytest.mark.parametrize("H,group,dh,past,new", [
    (1, 1, 128, [4200, 70], [1, 1]),               # pages by windows of 64, shares of the keys
    (2, 3, 64, [3000], [11]),
    (1, 2, 128, [2500, 2111], [130, 1]),           # many queries and shares
    (1, 1, 64, [2049], [300]),
])
def test_rows_of_many_pages(elem, H, group, dh, past, new):
    c = Case(elem, H, dh, 32, past, new, seed=H + dh + new[0])
    q = torch.randn(sum(new), H * group, dh, generator=torch.Generator().manual_seed(12)).bfloat16().cuda()
    c.append([0] * len(past), past)
    c.check(q, c.attend(q, files=True))
    assert torch.equal(c.attend(q), c.attend(q))


@pytest.mark.parametrize("elem", [R.BF16, R.FP8])
@pytest.mark.parametrize("dh", [64, 128])
@pytest.mark.parametrize("new", [1, 9, 150])
def test_positions_without_a_page(elem, dh, new):
    """Holes in the block table: first, last, in the middle, several in a row, two windows of 64 pages on."""
    past, H, group, scale = [2300, 500], 2, 2, 0.1
    c = Case(elem, H, dh, 32, past, [new, new], seed=dh + new)
    c.append([0, 0], c.total)
    table, lost = c.table.clone(), [[0, 7, 8, 9, 70, c.total[0] // 32], [3]]
    for r in range(2):
        for i in lost[r]:
            if i < table.shape[1]:
                table[r, i] = -1 - i if i % 2 else c.pool.shape[0] + i
    cache = skd.KvCache(c.pool, table.cuda(), H, dh, 32, elem)
    ch = c.chunk(past, [new, new])
    q = torch.randn(2 * new, H * group, dh, generator=torch.Generator().manual_seed(13)).bfloat16().cuda()
    out = torch.full_like(q, 5.0)
    cache.attend(ch, q, out, scale, workspace=torch.empty(cache.attend_workspace(ch, H * group), dtype=torch.uint8, device="cuda"))
    for r in range(2):
        has = torch.tensor([i // 32 not in lost[r] for i in range(c.total[r])])
        k, v = (torch.from_numpy(R.as_held(x[r].double().numpy(), elem)) for x in (c.k, c.v))
        for i in sorted({0, 1, new // 2, new - 1} & set(range(new))):
            n = past[r] + i + 1
            at = has[:n].nonzero()[:, 0]
            # one query that sees the positions left: attention() of its last position
            ref, bound = R.attention(q[r * new + i].cpu().double()[None], k[at], v[at], len(at) - 1, scale)
            assert ((out[r * new + i].cpu().double() - ref[0]).abs() <= bound[0]).all(), (r, i)


@pytest.mark.parametrize("elem", [R.BF16, R.FP8])
@pytest.mark.parametrize("past,new", [(40, 200), (1500, 140)])
def test_infinities_among_many_queries(elem, past, new):
    """Values that are not finite in the middle of a chunk: the queries before them stay finite, bit by bit what they are without."""
    H, dh = 1, 128
    c = Case(elem, H, dh, 64, [past], [new], seed=17)
    q = torch.randn(new, 2, dh, generator=torch.Generator().manual_seed(14)).bfloat16().cuda()
    at = past + new // 2 + 1
    c.append([0], c.total)
    clean = c.attend(q)
    c.check(q, clean)
    c.v[0][at, 0, 5], c.v[0][at + 3, 0, 6], c.v[0][at + 5, 0, 7] = math.inf, -math.inf, math.nan
    c.append([0], c.total)
    out = c.attend(q)
    seen = torch.arange(past, past + new) >= at
    assert torch.isfinite(out[~seen].float()).all()
    # (formed in two passes, the sums are rounded in another order)
    assert ((out - clean)[~seen].float().abs() <= 2.0 ** -6 * clean[~seen].float().abs() + 2.0 ** -8).all()
    for e, x, p in ((5, math.inf, at), (6, -math.inf, at + 3), (7, math.nan, at + 5)):
        col = out[torch.arange(past, past + new) >= p][..., e].float()
        if elem == R.BF16 and not math.isnan(x):
            assert (col == x).all()
        elif elem == R.BF16:
            assert torch.isnan(col).all()
        else:                                                         # 8 bits: the head's whole token reads as NaN
            assert torch.isnan(out[torch.arange(past, past + new) >= p].float()).all()


@pytest.mark.parametrize("elem", [R.BF16, R.FP8])
@pytest.mark.parametrize("group,dh,new", [(40, 128, 1), (70, 64, 1), (130, 128, 1), (33, 64, 4)])
def test_many_query_heads_of_a_kv_head(elem, group, dh, new):
    c = Case(elem, 2, dh, 64, [130, 0, 63], [new, 1, new], seed=group)
    q = torch.randn(2 * new + 1, 2 * group, dh, generator=torch.Generator().manual_seed(15)).bfloat16().cuda()
    c.append([0] * 3, c.past)
    c.check(q, c.attend(q, files=True))


@pytest.mark.parametrize("elem", [R.BF16, R.FP8])
@pytest.mark.parametrize("past,new", [([70, 5], [1, 1]), ([40, 0], [20, 3]), ([300, 20], [140, 70])])
def test_queries_and_outputs_with_strides(elem, past, new):
    """q, k and v side by side in one array, outputs in another with room between the tokens, which stays as it was."""
    H, group, dh = 2, 2, 64
    c = Case(elem, H, dh, 32, past, new, seed=new[0])
    T, W = sum(new), H * dh
    packed = torch.full((T, (group + 2) * W + 24), 9.0, dtype=torch.bfloat16, device="cuda")
    q = torch.randn(T, group * W, generator=torch.Generator().manual_seed(16)).bfloat16().cuda()
    packed[:, :group * W], packed[:, group * W:(group + 1) * W], packed[:, (group + 1) * W:(group + 2) * W] = q, c.tokens(c.k, past, new).flatten(1), c.tokens(c.v, past, new).flatten(1)
    c.append([0, 0], past)
    out = torch.full((T, group * W + 40), 5.0, dtype=torch.bfloat16, device="cuda")
    ch = c.chunk(past, new)
    c.cache.attend(ch, packed[:, :group * W], out[:, 8:8 + group * W], 0.125, packed[:, group * W:(group + 1) * W], packed[:, (group + 1) * W:(group + 2) * W],
                   workspace=torch.empty(c.cache.attend_workspace(ch, H * group), dtype=torch.uint8, device="cuda"))
    c.check(q.view(T, H * group, dh), out[:, 8:8 + group * W].reshape(T, H * group, dh).cpu())
    assert (out[:, :8] == 5).all() and (out[:, 8 + group * W:] == 5).all()


@pytest.mark.parametrize("elem", [R.BF16, R.FP8])
@pytest.mark.parametrize("new", [1, 6, 150])
def test_queries_that_are_not_finite(elem, new):
    """They are NaN by themselves: the queries beside them are what they are without."""
    c = Case(elem, 1, 128, 64, [200], [new], seed=new)
    q = torch.randn(new, 4, 128, generator=torch.Generator().manual_seed(18)).bfloat16().cuda()
    c.append([0], c.total)
    bad = q.clone()
    bad[new // 2, 1, 3], bad[new - 1, 3, 9] = math.nan, math.inf
    out = c.attend(bad)
    odd = torch.zeros(new, 4, dtype=torch.bool)
    odd[new // 2, 1] = odd[new - 1, 3] = True
    assert torch.isnan(out[odd].float()).all()
    k, v = (torch.from_numpy(R.as_held(x[0].double().numpy(), elem)) for x in (c.k, c.v))
    ref, bound = R.attention(q.cpu().double(), k, v, 200, 1 / math.sqrt(128))
    assert ((out.double() - ref).abs() <= bound)[~odd].all()


def test_bounds_that_are_too_small_or_too_large():
    """max_past only decides how the work is shared out; tokens beyond max_new are left out."""
    c = Case(R.BF16, 2, 64, 32, [2000, 64], [3, 3], seed=5)
    c.append([0, 0], c.total)
    q = torch.randn(6, 2, 64, generator=torch.Generator().manual_seed(19)).bfloat16().cuda()
    for max_past in (0, 1999, 1 << 29):
        ch = skd.KvChunk(i32([0, 3, 6]), i32([2000, 64]), 6, 3, max_past)
        out = torch.full_like(q, 5.0)
        c.cache.attend(ch, q, out, 0.125, workspace=torch.empty(c.cache.attend_workspace(ch, 2), dtype=torch.uint8, device="cuda"))
        c.check(q, out.cpu())
    ch = skd.KvChunk(i32([0, 3, 6]), i32([2000, 64]), 6, 2, 2000)
    out = torch.full_like(q, 5.0)
    c.cache.attend(ch, q, out, 0.125, workspace=torch.empty(c.cache.attend_workspace(ch, 2), dtype=torch.uint8, device="cuda"))
    assert (out[[2, 5]] == 5).all() and (out[[0, 1, 3, 4]] != 5).any(-1).all()


def test_two_streams_at_once():
    """Rows of one pool that share no page, on two streams with workspaces of their own, again and again."""
    c = Case(R.FP8, 2, 128, 64, [3000, 2500], [1, 1], seed=23)
    c.append([0, 0], c.total)
    q = torch.randn(2, 8, 128, generator=torch.Generator().manual_seed(20)).bfloat16().cuda()
    z, u = torch.randn(2, 60000, generator=torch.Generator().manual_seed(21)).cuda(), torch.tensor([0.3, 0.8]).cuda()
    parts = []
    for r in range(2):
        cache = skd.KvCache(c.pool, c.table[r:r + 1].cuda(), 2, 128, 64, R.FP8)
        ch = skd.KvChunk(i32([0, 1]), i32([c.past[r]]), 1, 1, 3000)
        ws = [torch.empty(n, dtype=torch.uint8, device="cuda") for n in (cache.attend_workspace(ch, 8), skd.sample_workspace(1, 60000))]
        parts.append((torch.cuda.Stream(), cache, ch, q[r:r + 1], torch.zeros(20, 8, 128, dtype=torch.bfloat16, device="cuda"), z[r:r + 1], u[r:r + 1],
                      torch.zeros(20, dtype=torch.int32, device="cuda"), torch.full((1,), 0.9, device="cuda"), *ws))
    kv = [(c.tokens(c.k, c.past, c.new)[r:r + 1].contiguous(), c.tokens(c.v, c.past, c.new)[r:r + 1].contiguous()) for r in range(2)]
    torch.cuda.synchronize()
    for i in range(20):
        for r, (s, cache, ch, qr, out, zr, ur, tok, top_p, ws, draw_ws) in enumerate(parts):
            cache.attend(ch, qr, out[i:i + 1], 1 / math.sqrt(128), *kv[r], workspace=ws, stream=s.cuda_stream)
            skd.sample(zr, ur, tok[i:i + 1], top_p=top_p, workspace=draw_ws, stream=s.cuda_stream)
    torch.cuda.synchronize()
    for r in range(2):
        out, tok = parts[r][4], parts[r][7]
        assert (out == out[0]).all() and (tok == tok[0]).all()
        assert int(tok[0]) == reference(z[r].cpu().numpy(), float(u[r]), p=float(np.float32(0.9)))
    c.check(q, torch.cat([parts[0][4][:1], parts[1][4][:1]]).cpu())

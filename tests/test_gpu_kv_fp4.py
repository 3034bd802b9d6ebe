"""Pages of 4 bits: keys and values filed, read back and attended to (SKD_KV_FP4), against 64 bits on the CPU."""
import math

import numpy as np
import pytest
import torch

import kv_scores_reference as S
from paper_2307_02628_amd import skd

pytestmark = pytest.mark.gpu

LENGTHS = [([0], [1]), ([0, 5], [3, 0]), ([0, 31, 32, 33, 100, 0], [33, 1, 32, 64, 29, 1]), ([63, 1, 7], [1, 1, 1]), ([2, 30], [8, 9])]


@pytest.mark.parametrize("H,dh,page", [(1, 64, 32), (3, 128, 64), (2, 64, 96), (5, 128, 128)])
@pytest.mark.parametrize("past,new", LENGTHS)
def test_filed_and_read_back(H, dh, page, past, new):
    c = S.Rows(S.FP4, H, dh, page, past, new, seed=H + dh)
    zero = [0] * len(past)
    if max(past):
        c.append(zero, past)
    c.append(past, new)
    k, v = c.read(zero, c.total)
    assert torch.equal(k.double(), c.held(c.k, zero, c.total)) and torch.equal(v.double(), c.held(c.v, zero, c.total))
    k16, v16 = c.read(past, new, torch.bfloat16)                    # only the new ones, as bf16: exact too
    assert torch.equal(k16.double(), c.held(c.k, past, new)) and torch.equal(v16.double(), c.held(c.v, past, new))
    # the pages as documented, and nothing written where no token went
    pool = c.pool.cpu().numpy()
    for r, t in enumerate(c.total):
        for i in range(c.table.shape[1]):
            n = min(max(t - i * page, 0), page)
            if n == 0:
                continue
            K, V = S.unpack_page4(pool[c.table[r, i]], H, dh, page)
            for got, x in ((K, c.k), (V, c.v)):
                np.testing.assert_array_equal(got[:n], S.as_held(x[r][i * page:i * page + n].double().numpy(), S.FP4))
                assert np.isnan(got[n:]).all()
    assert (c.pool[-1] == 255).all()


@pytest.mark.parametrize("tokens", [5, 40])                         # by tokens, by blocks
def test_values_at_the_ends_of_the_range(tokens):
    for part in range(8 if tokens == 5 else 1):
        c = S.Rows(S.FP4, 2, 64, 32, [0], [40], seed=3)
        k = c.k[0]
        k[0] = 0.0
        k[1] = -0.0
        k[2, 0, 5] = float("inf")
        k[3, 1, 63] = float("-inf")
        k[4, 0, 0] = float("nan")
        k[5] *= 2.0 ** -140                                          # below what the smallest exponent reaches
        k[6] *= 2.0 ** -125
        k[7, 0, 0] = torch.finfo(torch.bfloat16).max                 # the largest exponent: codes end at 3
        k[7, 1] = torch.finfo(torch.bfloat16).max * torch.linspace(-1, 1, 64)
        k[8, 0] = 6.0
        k[9, 0] = 6.0625                                             # the next power of two
        k[10, 0] = torch.tensor([6.0 * 2.0 ** -(i % 7) for i in range(64)]).bfloat16()
        k[11, 1] = torch.tensor([6.0, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 0.2490234375, 0.251953125, 4.96875, 5.03125, 1.0, 3.0, 2.0, 0.5] * 4).bfloat16()  # halves
        k[12, 0] = -k[11, 1]
        k[13, 0, :32], k[13, 0, 32:] = 2.0 ** 60, 2.0 ** -60         # an exponent for each 32
        c.v[0][:] = k.roll(1, 1)
        at = 5 * part if tokens == 5 else 0
        c.append([at], [tokens])
        for got, x in zip(c.read([at], [tokens]), (c.k, c.v)):
            want = c.held(x, [at], [tokens])
            assert torch.equal(torch.isnan(got), torch.isnan(want))
            assert torch.equal(torch.nan_to_num(got.double(), nan=1.0), torch.nan_to_num(want, nan=1.0))


def test_strided_tokens_and_pages_that_are_none():
    c = S.Rows(S.FP4, 2, 64, 32, [10, 40, 0], [30, 30, 20], seed=5, spare=2)
    T, W = 80, 2 * 64
    packed = torch.full((T, 3 * W + 8), 9.0, dtype=torch.bfloat16, device="cuda")
    packed[:, W:2 * W] = c.tokens(c.k, c.past, c.new).flatten(1)
    packed[:, 2 * W:3 * W] = c.tokens(c.v, c.past, c.new).flatten(1)
    lost = c.table.clone()
    lost[1, 1], lost[2, 0] = -7, c.pool.shape[0]
    cache = skd.KvCache(c.pool, lost.cuda(), 2, 64, 32, S.FP4)
    before = c.pool.clone()
    cache.append(c.chunk(c.past, c.new), packed[:, W:2 * W], packed[:, 2 * W:3 * W])
    k, v = c.read(c.past, c.new)
    want = c.held(c.k, c.past, c.new)
    assert torch.equal(k[:30].double(), want[:30]) and torch.equal(k[54:60].double(), want[54:60])
    for r, i in ((1, 1), (2, 0)):
        assert torch.equal(c.pool[c.table[r, i]], before[c.table[r, i]])
    assert torch.equal(c.pool[-1], before[-1])
    ko, vo = (torch.full((T, 2, 64), 7.0, device="cuda") for _ in range(2))
    cache.read(c.chunk(c.past, c.new), ko, vo)
    assert (ko[30:54] == 7).all() and (vo[60:] == 7).all() and torch.equal(ko[:30].cpu().double(), want[:30])


ATTEND = [
    # H, group, dh, page, past, new
    (4, 1, 64, 64, [31, 20], [1, 1]),
    (2, 1, 128, 64, [0, 64, 33, 700], [1, 1, 1, 1]),
    (3, 4, 128, 32, [100, 0, 1500], [1, 1, 1]),
    (1, 8, 64, 96, [5, 40], [3, 2]),
    (2, 3, 128, 64, [0, 63, 17], [5, 7, 0]),
    (2, 20, 64, 64, [70, 2], [1, 1]),                                # a group wider than a tile
    (1, 8, 128, 64, [1000], [1]),
    (2, 1, 128, 64, [0, 300, 9], [70, 33, 1]),
    (1, 2, 64, 128, [130, 0], [129, 64]),
    (2, 2, 128, 64, [1000, 31], [200, 257]),
    (2, 1, 64, 32, [500, 2000], [130, 90]),
]


@pytest.mark.parametrize("H,group,dh,page,past,new", ATTEND)
def test_attention(H, group, dh, page, past, new):
    c = S.Rows(S.FP4, H, dh, page, past, new, seed=11 + group, spare=1)
    q = torch.randn(sum(new), H * group, dh, generator=torch.Generator().manual_seed(1)).bfloat16().cuda()
    if max(past):
        c.append([0] * len(past), past)
    out = c.attend(q, files=True)
    c.check(q, out)
    assert torch.equal(c.attend(q), out) or max(new) == 1            # the cache holds the tokens now
    c.check(q, c.attend(q))
    k, v = c.read([0] * len(past), c.total)
    assert torch.equal(k.double(), c.held(c.k, [0] * len(past), c.total)) and torch.equal(v.double(), c.held(c.v, [0] * len(past), c.total))


@pytest.mark.parametrize("fill", [0xfd, 0xfe, 0x7f, 0x00])
@pytest.mark.parametrize("past,new", [([31, 20], [1, 1]), ([100, 0], [9, 4]), ([3, 40], [70, 33]), ([1000, 31], [200, 257])])
def test_places_that_nobody_wrote_may_hold_anything(fill, past, new):
    c = S.Rows(S.FP4, 2, 128, 96, past, new, seed=17, spare=1, fill=fill)
    q = torch.randn(sum(new), 4, 128, generator=torch.Generator().manual_seed(1)).bfloat16().cuda()
    c.append([0, 0], past)
    c.check(q, c.attend(q, files=True))
    c.check(q, c.attend(q, window=20), window=20)


@pytest.mark.parametrize("scale,size", [(0.01, 1.0), (1.0, 1.0), (0.125, 8.0)])
def test_attention_of_flat_and_sharp_scores(scale, size):
    c = S.Rows(S.FP4, 2, 64, 64, [200, 65], [40, 33], seed=21)
    q = (size * torch.randn(73, 4, 64, generator=torch.Generator().manual_seed(2))).bfloat16().cuda()
    c.append([0, 0], c.total)
    c.check(q, c.attend(q, scale=scale), scale)


@pytest.mark.parametrize("size", [2.0 ** -118, 2.0 ** 100])
def test_attention_to_values_at_the_ends(size):
    c = S.Rows(S.FP4, 1, 128, 32, [70, 3], [1, 2], seed=23)
    for v in c.v:
        v *= size
    q = torch.randn(3, 2, 128, generator=torch.Generator().manual_seed(2)).bfloat16().cuda()
    c.append([0, 0], c.total)
    out = c.attend(q)
    c.v = [x / size for x in c.v]                                    # (exact, and so is what is held)
    c.check(q, out.double() / size)


@pytest.mark.parametrize("new", [1, 20, 130])
def test_attention_to_the_largest_values(new):
    """Exponents of 126, whose codes end at 3: finite where they are seen and where they are not."""
    c = S.Rows(S.FP4, 1, 64, 32, [40], [new], seed=27)
    big = torch.finfo(torch.bfloat16).max
    c.v[0][41:] = torch.where(c.v[0][41:] > 0, big, -big)
    c.append([0], c.total)
    q = torch.randn(new, 2, 64, generator=torch.Generator().manual_seed(2)).bfloat16().cuda()
    out = c.attend(q, window=1)                                      # each token's own value, as it is held
    want = c.held(c.v, c.past, c.new)[:, :1].expand(-1, 2, -1)
    assert torch.equal(out.double(), want)
    first = c.attend(q, end=[41] * new)                              # those before alone
    c.check(q, first, end=[41] * new)


@pytest.mark.parametrize("new", [1, 4, 70])
def test_infinities_that_a_query_does_not_see(new):
    """What is not finite at a position reaches the queries from that position on, and no other, in the 32 elements around it."""
    c = S.Rows(S.FP4, 2, 64, 64, [40, 10], [new, new], seed=31)
    if new > 1:
        at = 40 + new - 2
        c.v[0][at, 0, 3] = float("inf")
        c.v[0][at, 1, 37] = float("nan")
        c.v[0][at + 1, 0, 40] = float("-inf")
        c.k[1][10 + new - 1, 1, 0] = float("nan")
    else:
        c.v[0][40, 0, 3] = float("inf")
    q = torch.randn(2 * new, 4, 64, generator=torch.Generator().manual_seed(3)).bfloat16().cuda()
    c.append([0, 0], c.past)
    for files in (True, False):
        out = c.attend(q, files=files).double()
        for r in range(2):
            k, v = (torch.from_numpy(S.as_held(x[r].double().numpy(), S.FP4)) for x in (c.k, c.v))
            for i in range(new):
                n = c.past[r] + i + 1
                for h in range(4):
                    w = torch.softmax(q[r * new + i, h].cpu().double() @ k[:n, h // 2].t() / 8, -1)
                    ref, got = (w[:, None] * v[:n, h // 2]).sum(0), out[r * new + i, h]
                    assert torch.equal(torch.isnan(got), torch.isnan(ref)), (files, r, i, h)
                    ok = torch.isfinite(ref)
                    # (the bound of the reference, coarser: |v| is below 8)
                    assert ((got - ref)[ok].abs() <= 2.0 ** -7 * 8).all()


def test_rows_without_pages_and_rows_behind_the_last():
    c = S.Rows(S.FP4, 2, 64, 32, [40, 20], [2, 3], seed=41)
    c.append([0, 0], c.total)
    none = skd.KvCache(c.pool, torch.full_like(c.table, -1).cuda(), 2, 64, 32, S.FP4)
    q = torch.randn(8, 2, 64, generator=torch.Generator().manual_seed(3)).bfloat16().cuda()
    ch = skd.KvChunk(torch.tensor([0, 2, 5], dtype=torch.int32, device="cuda"), torch.tensor([40, 20], dtype=torch.int32, device="cuda"), 8, 3, 40)
    out = torch.full_like(q, 3.0)
    ws = torch.empty(c.cache.attend_workspace(ch, 2), dtype=torch.uint8, device="cuda")
    c.cache.attend(ch, q, out, 0.125, workspace=ws)
    c.check(q[:5], out[:5].cpu())
    assert (out[5:] == 3).all()
    none.attend(ch, q, out, 0.125, workspace=ws)
    assert (out[:5] == 0).all() and (out[5:] == 3).all()


def test_holes_in_the_block_table_among_many_queries():
    c = S.Rows(S.FP4, 2, 128, 32, [0], [200], seed=43, spare=1)
    c.append([0], [200])
    lost = c.table.clone()
    lost[0, 2] = -1                                                  # positions 64 .. 95
    cache = skd.KvCache(c.pool, lost.cuda(), 2, 128, 32, S.FP4)
    q = torch.randn(200, 2, 128, generator=torch.Generator().manual_seed(3)).bfloat16().cuda()
    ch, out = c.chunk([0], [200]), torch.zeros_like(q)
    cache.attend(ch, q, out, 0.1, workspace=torch.empty(cache.attend_workspace(ch, 2), dtype=torch.uint8, device="cuda"))
    k, v = (torch.from_numpy(S.as_held(x[0].double().numpy(), S.FP4)) for x in (c.k, c.v))
    keep = torch.tensor([i for i in range(200) if not 64 <= i < 96])
    for i in (0, 63, 64, 95, 96, 199):
        seen = keep[keep <= i]
        ref, bound = S.attention(q[i:i + 1].cpu().double(), k[seen], v[seen], len(seen) - 1, 0.1)
        assert ((out[i:i + 1].cpu().double() - ref).abs() <= bound).all(), i


def test_pages_beyond_32_bits():
    H, dh, page = 32, 128, 4096
    size = H * page // 32 * 34 * dh                                   # 17 MiB a page
    pages = (9 << 29) // size + 3                                     # 4.5 GiB
    pool = torch.empty(pages, size, dtype=torch.uint8, device="cuda")
    table = torch.tensor([[pages - 1, 0, pages - 2]], dtype=torch.int32, device="cuda")
    cache = skd.KvCache(pool, table, H, dh, page, S.FP4)
    g = torch.Generator(device="cuda").manual_seed(1)
    n = 2 * page + 77
    k, v = (torch.randn(n, H, dh, generator=g, device="cuda").bfloat16() for _ in range(2))
    every, zero = torch.tensor([0, n], dtype=torch.int32, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
    cache.append(skd.KvChunk(every, zero, n, n, 0), k, v)
    ko, vo = torch.empty_like(k), torch.empty_like(v)
    cache.read(skd.KvChunk(every, zero, n, n, 0), ko, vo)
    kh, vh = (torch.from_numpy(S.as_held(x.cpu().double().numpy(), S.FP4)) for x in (k, v))
    assert torch.equal(kh, ko.cpu().double()) and torch.equal(vh, vo.cpu().double())
    q = torch.randn(1, H, dh, generator=g, device="cuda").bfloat16()
    ch = skd.KvChunk(torch.tensor([0, 1], dtype=torch.int32, device="cuda"), torch.tensor([n - 1], dtype=torch.int32, device="cuda"), 1, 1, n)
    out = torch.empty_like(q)
    cache.attend(ch, q, out, 1 / math.sqrt(dh), workspace=torch.empty(cache.attend_workspace(ch, H), dtype=torch.uint8, device="cuda"))
    ref, bound = S.attention(q.cpu().double(), kh, vh, n - 1, 1 / math.sqrt(dh))
    assert ((out.cpu().double() - ref).abs() <= bound).all()

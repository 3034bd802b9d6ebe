"""The paged cache at its edges: new tokens whose positions have no page, values at the small end of the range, rows in many shares,
workspaces that are refused, layers of a state that are set to nothing."""
import math

import numpy as np
import pytest
import torch

import kv_reference as R
from paper_2307_02628_amd import skd
from test_gpu_decode_chunk import NARROW, Run
from test_gpu_kv_ops import Case

pytestmark = pytest.mark.gpu


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def attended(c, cache, ch, q, out, scale, kv=()):
    ws = torch.empty(cache.attend_workspace(ch, q.shape[1]), dtype=torch.uint8, device="cuda")
    cache.attend(ch, q, out, scale, *kv, workspace=ws)
    return out.cpu()


@pytest.mark.parametrize("elem", [R.BF16, R.FP8])
@pytest.mark.parametrize("H,group,dh", [(2, 1, 64), (1, 4, 128), (2, 16, 128), (1, 20, 64)])
@pytest.mark.parametrize("long", [0, 4000])
def test_a_new_token_without_a_page(elem, H, group, dh, long):
    """One token a row, filed by the call that attends to it: without a page it is dropped and nobody sees it, as if it had been
    filed by a call of its own."""
    page, scale = 32, 0.2
    past = [64 + long, 0, 96 + long, 40, 70]
    c = Case(elem, H, dh, page, past, [1] * 5, seed=dh + group)
    c.append([0] * 5, past)
    width = (96 + long) // page
    table = c.table[:, :width].clone()                                # row 2 is full: its new position is behind its pages
    table[0, past[0] // page] = -1
    table[1, 0] = -5                                                  # row 1 holds nothing at all
    table[3, 1] = c.pool.shape[0]
    cache = skd.KvCache(c.pool, table.cuda(), H, dh, page, elem)
    ch = c.chunk(past, [1] * 5)
    q = torch.randn(5, H * group, dh, generator=torch.Generator().manual_seed(31)).bfloat16().cuda()
    kv = c.tokens(c.k, past, [1] * 5), c.tokens(c.v, past, [1] * 5)
    before = c.pool.clone()
    out = attended(c, cache, ch, q, torch.full_like(q, 5.0), scale, kv)
    after = c.pool.clone()
    c.pool.copy_(before)
    cache.append(ch, *kv)
    assert torch.equal(after.view(torch.uint8), c.pool.view(torch.uint8))
    apart = attended(c, cache, ch, q, torch.full_like(q, 5.0), scale)
    for r in range(5):
        has = torch.tensor([i // page < width and 0 <= table[r, i // page] < c.pool.shape[0] for i in range(past[r] + 1)])
        assert bool(has[-1]) == (r == 4)
        at = has.nonzero()[:, 0]
        for got in (out[r], apart[r]):
            if len(at) == 0:
                assert (got == 0).all()
                continue
            k, v = (torch.from_numpy(R.as_held(x[r][at].double().numpy(), elem)) for x in (c.k, c.v))
            ref, bound = R.attention(q[r:r + 1].cpu().double(), k, v, len(at) - 1, scale)
            assert ((got.double() - ref[0]).abs() <= bound[0]).all(), r


@pytest.mark.parametrize("elem", [R.BF16, R.FP8])
@pytest.mark.parametrize("H,group,new", [(1, 1, 1), (1, 8, 1), (2, 3, 5), (1, 2, 14)])
def test_64_wide_heads_in_many_shares(elem, H, group, new):
    c = Case(elem, H, 64, 32, [9000], [new], seed=group + new)
    q = torch.randn(new, H * group, 64, generator=torch.Generator().manual_seed(32)).bfloat16().cuda()
    shares = c.cache.attend_workspace(c.chunk(c.past, c.new), H * group) / (4 * 66 * new * H * group)
    assert shares > 8
    c.append([0], c.past)
    c.check(q, c.attend(q, files=True))
    c.check(q, c.attend(q))


@pytest.mark.parametrize("dh", [64, 128])
@pytest.mark.parametrize("past,new", [(4, 1), (300, 1), (70, 20), (500, 150)])
@pytest.mark.parametrize("files", [True, False])
def test_values_of_the_smallest_exponent(dh, past, new, files):
    """8-bit values whose exponent byte is 0 (2^-127) count for what they are, in the call that files them and afterwards."""
    c = Case(R.FP8, 1, dh, 64, [past], [new], seed=past)
    g = torch.Generator().manual_seed(33)
    c.v[0][:] = (torch.randint(8, 16, c.v[0].shape, generator=g) * 2.0 ** -123).bfloat16()  # 128 .. 240 units of 2^-127: exact
    c.k[0][:] = torch.rand(c.k[0].shape, generator=g).bfloat16() - 0.5
    q = ((torch.rand(new, 2, dh, generator=g) - 0.5) / 8).bfloat16().cuda()
    c.append([0], [past])
    if not files:
        c.append([past], [new])
    out = c.attend(q, files=files, scale=0.125).double()
    k = torch.from_numpy(R.as_held(c.k[0].double().numpy(), R.FP8))
    ref, bound = R.attention(q.cpu().double(), k, c.v[0].double(), past, 0.125)
    # Beside the bound of attention(): a weight times 2^-127 is rounded to a multiple of 2^-133, by 2^-134 at most, and a code is 240 at
    # most: each key adds 2^-126, over a sum of the weights that is 1/2 at least for each (scores are below 0.125 * dh / 2 / 16 <= 1/2
    # in magnitude: weights lie within a factor of e of each other, and one of them is at least 1).
    allowed = bound + 2.0 ** -126 * math.e
    assert allowed.max() < ref.min() / 2
    assert ((out - ref).abs() <= allowed).all()


@pytest.mark.parametrize("past,new", [(40, 1), (70, 20), (500, 150)])
def test_keys_of_the_smallest_exponent(past, new):
    """Tiny keys against huge queries: scores of ordinary size."""
    c = Case(R.FP8, 1, 128, 64, [past], [new], seed=past)
    g = torch.Generator().manual_seed(34)
    c.k[0][:] = ((torch.randint(0, 9, c.k[0].shape, generator=g) - 4) * 2.0 ** -122).bfloat16()
    q = (torch.randn(new, 2, 128, generator=g) * 2.0 ** 120).bfloat16().cuda()
    c.append([0], c.total)
    c.check(q, c.attend(q, scale=0.125), 0.125)


def test_workspaces_that_are_refused():
    c = Case(R.BF16, 2, 64, 32, [3], [1], seed=71, spare=3999)
    ch, lib = c.chunk([100000], [1]), skd.lib()
    need = c.cache.attend_workspace(ch, 2)
    assert need > 0
    dev, host = torch.zeros(1, 2, 64, dtype=torch.bfloat16, device="cuda"), torch.zeros(need, dtype=torch.uint8)
    ws = torch.empty(need, dtype=torch.uint8, device="cuda")

    def rc(p, n):
        return lib.skd_kv_attend(c.cache.ref, ch.ref, 2, 0.1, dev.data_ptr(), 128, None, 0, None, 0, dev.data_ptr(), 128, p, n, None)

    assert rc(None, need) == rc(None, 0) == skd.ERR_NULL
    assert rc(ws.data_ptr(), need - 1) == skd.ERR_NOMEM
    at = -host.data_ptr() % 16                                        # (an aligned place in ordinary host memory)
    assert rc(host.data_ptr() + at, need) == skd.ERR_RANGE


@pytest.mark.parametrize("dtype", [skd.BF16, skd.FP32, skd.BF16_KV8])
def test_layers_that_are_set_to_nothing(dtype):
    """Layers without arrays hold zeros, whatever the generation before has left there."""
    r = Run(NARROW, 3, 20, 60, NARROW.L, NARROW.L, 0, dtype, ragged=True)
    for t in range(20, 40):
        r.step(t)
    g = np.random.default_rng(5)
    K, V = ([g.standard_normal((3, 37, NARROW.d)).astype(np.float32) for _ in range(NARROW.L)] for _ in range(2))
    K[1] = V[1] = K[2] = V[3] = None
    r.dec.kv_load(37, K, V, r.start)
    for b in range(3):
        s = r.start[b]
        for l in range(NARROW.L):
            k, v = r.dec.kv_read(l, b)
            assert len(k) == 37
            assert ((k[s:] == 0).all() and (v[s:] == 0).all()) == (l > 0)
    r.step(37)
    assert np.isfinite(r.logits()).all()
    r.dec.close()


def test_temperatures_up_to_the_largest():
    r = Run(NARROW, 3, 5, 20, 1, 2)
    u = [0.1, 0.5, 0.9]
    for t, rc in ((np.finfo(np.float32).max, skd.OK), (3.2e38, skd.OK), (np.inf, skd.ERR_RANGE), (np.nan, skd.ERR_RANGE), (-1.0, skd.ERR_RANGE)):
        got, tok, _ = r.dec.logits_sample_rows_rc(u, temperature=[1.0, t, 1.0])
        assert got == rc
        if rc == skd.OK:
            assert tok[1] == NARROW.V // 2                            # every token alike: the one at which the running mass passes a half
    r.dec.close()


@pytest.mark.parametrize("elem", [R.BF16, R.FP8])
def test_one_long_row_among_many(elem):
    """More blocks, max_new of every row, than a launch has workgroups: the tokens of all rows are filed and read back."""
    rows, n, few, page, dh = 4110, 131000, 72, 64, 64
    assert (n + 62) // 32 * rows >= 2 ** 24
    table = torch.full((rows, -(-n // page)), -1, dtype=torch.int32)
    order = torch.randperm(table.shape[1] + 4, generator=torch.Generator().manual_seed(35)).int()
    table[7] = order[:table.shape[1]]
    table[rows - 1, :4] = order[table.shape[1]:]
    size = page * (4 * dh if elem == R.BF16 else 2 * dh + 2)
    pool = torch.zeros(len(order), size, dtype=torch.uint8, device="cuda")
    cache = skd.KvCache(pool, table.cuda(), 1, dh, page, elem)
    first = torch.zeros(rows + 1, dtype=torch.int32)
    first[8:], first[rows] = n, n + few
    past = torch.zeros(rows, dtype=torch.int32)
    past[rows - 1] = 150
    ch = skd.KvChunk(first.cuda(), past.cuda(), n + few, n, 150)
    k, v = (torch.randn(n + few, 1, dh, generator=torch.Generator(device="cuda").manual_seed(i), device="cuda").bfloat16() for i in range(2))
    cache.append(ch, k, v)
    ko, vo = torch.full_like(k, 7.0), torch.full_like(v, 7.0)
    cache.read(ch, ko, vo)
    for x, y in ((k, ko), (v, vo)):
        assert torch.equal(torch.from_numpy(R.as_held(x.cpu().double().numpy(), elem)), y.cpu().double())


@pytest.mark.parametrize("new", [1, 20, 150])
def test_scores_of_minus_infinity(new):
    """Keys at -infinity of a query have no weight; a query that sees no others gets zeros."""
    past, H, dh = [40, 100], 2, 64
    c = Case(R.BF16, H, dh, 32, past, [new, new], seed=36)
    q = torch.randn(2 * new, 4, dh, generator=torch.Generator().manual_seed(37)).bfloat16()
    q[..., 0] = 1.0
    q = q.cuda()
    c.k[0][:, :, 0] = -math.inf                                       # row 0: all of them
    c.k[1][::3, :, 0] = -math.inf
    c.append([0, 0], past)
    for files in (True, False):
        out = c.attend(q, files=files)
        assert (out[:new] == 0).all()
        for i in sorted({0, new // 2, new - 1}):
            at = torch.tensor([p for p in range(past[1] + i + 1) if p % 3])
            ref, bound = R.attention(q[new + i].cpu().double()[None], c.k[1][at].double(), c.v[1][at].double(), len(at) - 1, 1 / math.sqrt(dh))
            assert ((out[new + i].double() - ref[0]).abs() <= bound[0]).all(), i

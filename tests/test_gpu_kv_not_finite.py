"""Keys and values that are not finite in blocks that all queries of a tile see whole, with and without changed scores (skd_kv_attend,
skd_kv_attend_scores), against the definition; and windows of all that 32 bits hold."""
import pytest
import torch

import kv_scores_reference as S

pytestmark = pytest.mark.gpu
ELEMS = [S.BF16, S.FP8, S.FP4]
CHANGES = {"none": {}, "cap": dict(cap=10.0), "slopes": dict(slopes=True), "both": dict(cap=10.0, slopes=True), "masks": dict(end=True)}


def queries(tokens, heads, dh, seed=1):
    return torch.randn(tokens, heads, dh, generator=torch.Generator().manual_seed(seed)).bfloat16().cuda()


def held(c, x):
    return [torch.from_numpy(S.as_held(t.double().numpy(), c.elem)) for t in x]


def check(c, q, out, how):
    """Every position is seen by every query and weighs more than nothing: a value that is not finite is in all outputs of its element, and a key of
    NaN in all of its head.  The others as if such values were 0 (their own elements are not looked at)."""
    (k, ), (v, ) = held(c, c.k), held(c, c.v)
    group, new = q.shape[1] // c.H, c.new[0]
    seen = c.past[0] + 1                                             # by all queries
    lost = torch.isnan(k[:seen]).any(2).any(0).repeat_interleave(group)
    up, down, nan = (f(v[:seen]).any(0).repeat_interleave(group, 0)[None].expand(new, -1, -1) for f in (torch.isposinf, torch.isneginf, torch.isnan))
    clean = (torch.where(torch.isfinite(k), k, 0.0), torch.where(torch.isfinite(v), v, 0.0))
    ref, bound = S.attention(q.cpu().double(), *clean, c.past[0], 1 / 8 if c.dh == 64 else 128 ** -0.5, **how)
    nan = nan | (up & down) | lost[None, :, None]
    out = out.double()
    assert torch.equal(torch.isnan(out), nan)
    assert torch.equal(out.isposinf(), up & ~nan) and torch.equal(out.isneginf(), down & ~nan)
    fine = ~(nan | up | down)
    assert fine.any() and ((out - ref).abs() <= bound)[fine].all()


@pytest.mark.parametrize("name", CHANGES)
@pytest.mark.parametrize("elem", ELEMS)
@pytest.mark.parametrize("dh", [64, 128])
@pytest.mark.parametrize("new,group", [(1, 1), (1, 4), (20, 1), (17, 2), (200, 1), (150, 2)])
def test_in_blocks_that_all_queries_see(new, group, dh, elem, name):
    past, H = 300, 4                                                 # (one head has nothing of the kind)
    c = S.Rows(elem, H, dh, 64, [past], [new], seed=81)
    v = c.v[0]
    v[40, 0, 3], v[40, 0, 50], v[75, 0, 50], v[130, 0, 5] = float("inf"), float("-inf"), float("inf"), float("nan")
    v[200, 2, 40] = float("-inf")
    c.k[0][41, 1, 7] = float("nan")
    c.append([0], c.total)
    how = dict(CHANGES[name])
    if "slopes" in how:
        how["slopes"] = [0.01 * (h % 4) for h in range(H * group)]
    if "end" in how:
        how["end"] = [past + i + 1 for i in range(new)]
    q = queries(new, H * group, dh)
    for files in (False, True):
        check(c, q, c.attend(q, files=files, **how), how)


@pytest.mark.parametrize("elem", ELEMS)
@pytest.mark.parametrize("new", [1, 9, 40])
def test_in_shares_of_a_long_row(elem, new):
    """In a share of the keys that is joined with others."""
    c = S.Rows(elem, 2, 128, 64, [9000], [new], seed=83)
    c.v[0][4000, 0, 3], c.v[0][20, 0, 70] = float("inf"), float("nan")
    c.append([0], c.total)
    q = queries(new, 4, 128)
    for how in ({}, dict(slopes=[0.001, 0.0, 0.0005, 0.0001]), dict(cap=5.0)):
        check(c, q, c.attend(q, **how), how)


@pytest.mark.parametrize("elem", ELEMS)
@pytest.mark.parametrize("new", [1, 9, 140])
def test_the_largest_window_is_none(elem, new):
    c = S.Rows(elem, 2, 128, 64, [500], [new], seed=3)
    c.append([0], c.total)
    q = queries(new, 4, 128)
    out = c.attend(q, window=(1 << 31) - 1)
    c.check(q, out)
    assert torch.equal(out, c.attend(q, begin=[0] * new))

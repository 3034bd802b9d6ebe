"""Attention with masks over rows of which only what their tokens see was ever filed: what the pages hold at the other positions, before, between
and behind, does not reach a query, whatever it is (skd_kv_attend_scores), against 64 bits on the CPU."""
import copy

import pytest
import torch

import kv_scores_reference as S
from paper_2307_02628_amd import skd

pytestmark = pytest.mark.gpu

# bytes of the pages that nobody filed: e4m3 NaN of either sign (exponents 2^0 and NaN), 4-bit exponents of 126, 127 and NaN with codes of 6 or 4
FILLS = [(S.BF16, 0xff), (S.BF16, 0x7f), (S.FP8, 0x7f), (S.FP8, 0xff), (S.FP4, 0x7f), (S.FP4, 0xfd), (S.FP4, 0xfe), (S.FP4, 0xff)]


def queries(tokens, heads, dh, seed=1):
    return torch.randn(tokens, heads, dh, generator=torch.Generator().manual_seed(seed)).bfloat16().cuda()


def changes(name, past, new):
    """What the call asks for, and the positions below past that are filed for it."""
    at = [past + i for i in range(new)]
    if name == "window":                                             # the last ones, from inside of a block on
        return dict(window=45), range(past - 44, past)
    if name == "begin":
        return dict(begin=[past - 20 + i % 3 for i in range(new)], cap=20.0), range(past - 20, past)
    if name == "end":                                                # a piece far before the tokens, and not the tokens
        return dict(end=[90 - i % 4 for i in range(new)], begin=[70] * new), range(70, 90)
    # tokens of two kinds: in one block both sees another part of it, and a part in between is nobody's
    return dict(begin=[66 if i % 2 else 85 for i in range(new)], end=[74 if i % 2 else p + 1 for i, p in enumerate(at)], slopes=True), [*range(66, 74), *range(85, past)]


@pytest.mark.parametrize("name", ["window", "begin", "end", "between"])
@pytest.mark.parametrize("new,group", [(1, 1), (1, 5), (4, 5), (9, 1), (30, 1), (20, 3), (70, 1), (150, 2)])
@pytest.mark.parametrize("dh", [64, 128])
@pytest.mark.parametrize("elem,fill", FILLS)
def test_places_that_no_token_sees(elem, fill, dh, new, group, name):
    past, H = 130, 2
    c = S.Rows(elem, H, dh, 64, [past], [new], seed=61, spare=1)
    c.pool.view(torch.uint8).fill_(fill)
    how, filed = changes(name, past, new)
    if how.pop("slopes", False):
        how["slopes"] = [2.0 ** -(2 + h) for h in range(H * group)]
    runs = [[p for p in filed if p < 80], [p for p in filed if p >= 80]] if name == "between" else [list(filed)]
    for run in runs:
        c.append([run[0]], [len(run)])
    q = queries(new, H * group, dh)
    c.check(q, c.attend(q, files=True, **how), **how)
    c.check(q, c.attend(q, **how), **how)                            # the cache holds the tokens now


@pytest.mark.parametrize("elem,fill", FILLS)
@pytest.mark.parametrize("new", [1, 6, 40])
def test_places_that_no_token_sees_of_a_long_row_in_shares(elem, fill, new):
    past, window = 9000, 2000
    c = S.Rows(elem, 1, 128, 64, [past], [new], seed=67)
    c.pool.view(torch.uint8).fill_(fill)
    c.append([past - window + 1], [window - 1])
    q = queries(new, 4, 128)
    for how in (dict(window=window), dict(window=window, slopes=[0.1, 0.0, 0.01, 1.0], cap=30.0)):
        c.check(q, c.attend(q, files=True, **how), **how)


def finite(c):
    """The same rows with what a page holds as infinity or NaN as zeros."""
    same = copy.copy(c)
    held = [torch.from_numpy(S.as_held(x.double().numpy(), c.elem)) for x in c.v]
    same.v = [torch.where(torch.isfinite(h), x.double(), 0.0).bfloat16() for h, x in zip(held, c.v)]
    return same


@pytest.mark.parametrize("elem", [S.BF16, S.FP8, S.FP4])
@pytest.mark.parametrize("past", [20, 300])
@pytest.mark.parametrize("dh", [64, 128])
def test_a_filed_value_that_is_not_finite_and_weighs_nothing(elem, past, dh):
    """The token of the call has an infinity and a NaN among its values, and a key of every block a score so much larger that its weight is 0 in 32 bits:
    queries that see it get no finite result, whether the call files it or the cache holds it, and others are as if it were not there."""
    c = S.Rows(elem, 2, dh, 64, [past], [1], seed=71)
    q = queries(1, 2, dh)
    c.k[0][5:past:16] = 400.0 / dh ** 0.5 * q[0].cpu()               # a score of about 400
    c.v[0][5:past:16] = c.v[0][5].clone()
    c.v[0][past, 0, 3], c.v[0][past, 1, 40] = float("inf"), float("nan")
    c.append([0], [past])
    for how in (dict(cap=1000.0), dict(window=past), dict(slopes=[2.0 ** -9, 0.0]), dict(slopes=[0.0, 2.0 ** -9], cap=1000.0, end=[past + 1])):
        for files in (True, False):
            out = c.attend(q, files=files, **how)[0]
            lost = torch.isnan(torch.from_numpy(S.as_held(c.v[0][past].double().numpy(), elem))) | torch.isinf(c.v[0][past])
            assert lost.any() and torch.equal(~torch.isfinite(out), lost), (how, files)
            finite(c).check(q, torch.where(lost, torch.from_numpy(S.as_held(c.v[0][5].double().numpy(), elem)), out.double())[None], **how)
    for how in (dict(end=[past]), dict(end=[past], cap=1000.0, slopes=[0.5, 0.0])):
        for files in (True, False):
            c.check(q, c.attend(q, files=files, **how), **how)

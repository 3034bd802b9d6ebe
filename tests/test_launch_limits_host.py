"""Sizes at the end of what a launch can have (its threads are counted in 32 bits), on the CPU: the largest are accepted by the calls
that size a workspace, one more is refused before any device work."""
import ctypes as C
import os

import pytest

from paper_2307_02628_amd import _build, skd
from test_kv_ops_host import append, attend, chunk, kv, read


@pytest.fixture(scope="module", autouse=True)
def _built():
    if not os.path.exists(skd.LIB_PATH):
        _build.build(force=True)


@pytest.mark.parametrize("heads,new,most", [
    (1, 1, 2 ** 24 - 1),        # a tile of 16 queries, 4 waves
    (20, 1, 2 ** 23 - 1),       # of 32, 8 waves
    (200, 1, 2 ** 23 - 8),      # two of 128 each, on places for a multiple of 8 rows
])
def test_rows_of_an_attention(heads, new, most):
    def space(rows):
        return skd.lib().skd_kv_attend_workspace(C.byref(kv(kv_heads=1, rows=rows)), C.byref(chunk(tokens=1, max_new=new)), heads)

    assert space(most) == 0 and space(most + 1) == skd.ERR_RANGE and space(2 ** 31 - 1) == skd.ERR_RANGE
    bad = kv(kv_heads=1, rows=most + 1)
    assert attend(bad, chunk(tokens=1, max_new=new), heads, qs=heads * 128, os_=heads * 128) == skd.ERR_RANGE


def test_blocks_of_a_cache():
    """Rows x kv heads x blocks of the longest row: products beyond 64 bits too."""
    huge = dict(kv_heads=65536, rows=2 ** 31 - 1, page_tokens=32, max_pages=2 ** 25 - 1)
    width = 65536 * 128
    for new in (1, 2 ** 30):
        ch = chunk(tokens=2 ** 30, max_new=new)
        for call in (append, read):
            assert call(kv(**huge), ch, ks=width, vs=width) == skd.ERR_RANGE
        assert attend(kv(**huge), ch, 65536, qs=width, os_=width) == skd.ERR_RANGE


def test_columns_of_a_token():
    """Query heads are elements of a token in 32 bits."""
    one = dict(c=kv(kv_heads=1, rows=1), ch=chunk(tokens=1, max_new=1, max_past=31))
    for dh in (64, 128):
        one["c"].head_dim = dh
        most = 2 ** 31 // dh - 1
        assert skd.lib().skd_kv_attend_workspace(C.byref(one["c"]), C.byref(one["ch"]), most) >= 0
        for heads in (most + 1, 2 ** 31 - 129):
            assert skd.lib().skd_kv_attend_workspace(C.byref(one["c"]), C.byref(one["ch"]), heads) == skd.ERR_RANGE
            assert attend(**one, heads=heads, qs=heads * dh, os_=heads * dh) == skd.ERR_RANGE


def test_scales_at_the_ends():
    """Scores are scaled to units of log 2, which has to be finite: what passes is then refused for its workspace."""
    few = dict(c=kv(max_pages=2000, rows=1), ch=chunk(max_past=100000))
    for scale in (1e-45, 1e-38, 2.0 ** 126):
        assert attend(**few, scale=scale) == skd.ERR_NULL
    for scale in (2.5e38, 3.4e38):
        assert attend(**few, scale=scale) == skd.ERR_RANGE


@pytest.mark.parametrize("vocab,most", [(1000, 2 ** 22 - 1), (262144, 2 ** 20 - 1)])
def test_rows_of_a_draw(vocab, most):
    lib, P = skd.lib(), 1 << 20
    assert lib.skd_sample_workspace(most, vocab) > 0
    assert lib.skd_sample_workspace(most + 1, vocab) == skd.ERR_RANGE
    assert lib.skd_sample(P, vocab, most + 1, vocab, None, P, P, P, 1 << 62, None) == skd.ERR_RANGE

"""Refusals of the cache's and the draw's calls, on the CPU: every one is answered before any device work."""
import ctypes as C
import os

import pytest

from paper_2307_02628_amd import _build, skd

P = 1 << 20  # stands for device memory: nothing here gets as far as looking at it


@pytest.fixture(scope="module", autouse=True)
def _built():
    if not os.path.exists(skd.LIB_PATH):
        _build.build(force=True)


def kv(**changed):
    f = dict(elem=skd.KV_BF16, kv_heads=4, head_dim=128, page_tokens=64, pages=10, rows=3, max_pages=5, pool=P, block_table=P)
    return skd.Kv(**{**f, **changed})


def chunk(**changed):
    f = dict(tokens=7, max_new=4, max_past=100, first=P, past=P)
    return skd.Chunk(**{**f, **changed})


def append(c=None, ch=None, k=P, ks=512, v=P, vs=512):
    return skd.lib().skd_kv_append(C.byref(c or kv()), C.byref(ch or chunk()), k, ks, v, vs, None)


def read(c=None, ch=None, elem=skd.W_FP32, k=P, ks=512, v=P, vs=512):
    return skd.lib().skd_kv_read(C.byref(c or kv()), C.byref(ch or chunk()), elem, k, ks, v, vs, None)


def attend(c=None, ch=None, heads=8, scale=0.1, q=P, qs=1024, k=None, ks=0, v=None, vs=0, o=P, os_=1024, ws=None, n=0):
    return skd.lib().skd_kv_attend(C.byref(c or kv()), C.byref(ch or chunk()), heads, scale, q, qs, k, ks, v, vs, o, os_, ws, n, None)


BAD_KV = [dict(elem=2), dict(elem=-1), dict(head_dim=96), dict(head_dim=0), dict(page_tokens=0), dict(page_tokens=48), dict(page_tokens=-32), dict(kv_heads=0), dict(pages=0),
          dict(rows=-1), dict(max_pages=0)]


@pytest.mark.parametrize("bad", BAD_KV, ids=str)
def test_shapes(bad):
    lib = skd.lib()
    assert lib.skd_kv_page_bytes(C.byref(kv(**bad))) == skd.ERR_SHAPE
    assert append(kv(**bad)) == read(kv(**bad)) == attend(kv(**bad)) == skd.ERR_SHAPE
    assert lib.skd_kv_attend_workspace(C.byref(kv(**bad)), C.byref(chunk()), 8) == skd.ERR_SHAPE


def test_sizes():
    lib = skd.lib()
    assert lib.skd_kv_page_bytes(C.byref(kv())) == 4 * 64 * 2 * 128 * 2
    assert lib.skd_kv_page_bytes(C.byref(kv(elem=skd.KV_FP8))) == 4 * 64 * 2 * 129
    assert lib.skd_kv_page_bytes(C.byref(kv(kv_heads=32, page_tokens=1 << 20, max_pages=1))) == 32 * (1 << 20) * 512
    assert lib.skd_kv_attend_workspace(C.byref(kv()), C.byref(chunk()), 8) >= 0
    assert lib.skd_kv_attend_workspace(C.byref(kv()), C.byref(chunk(tokens=0)), 8) == 0


def test_pointers_and_ranges():
    lib = skd.lib()
    assert lib.skd_kv_page_bytes(None) == skd.ERR_NULL
    assert lib.skd_kv_append(None, C.byref(chunk()), P, 512, P, 512, None) == skd.ERR_NULL
    assert lib.skd_kv_append(C.byref(kv()), None, P, 512, P, 512, None) == skd.ERR_NULL
    for call in (append, read, attend):
        assert call(kv(pool=None)) == call(kv(block_table=None)) == call(None, chunk(first=None)) == call(None, chunk(past=None)) == skd.ERR_NULL
        assert call(kv(pool=P + 8)) == call(kv(block_table=P + 2)) == call(None, chunk(first=P + 1)) == call(None, chunk(past=P + 3)) == skd.ERR_SHAPE
        assert call(None, chunk(tokens=-1)) == call(None, chunk(max_new=-1)) == call(None, chunk(max_past=-1)) == skd.ERR_RANGE
        assert call(kv(max_pages=1 << 26)) == skd.ERR_RANGE           # positions beyond 32 bits
        assert call(None, chunk(max_new=0)) == call(None, chunk(tokens=0)) == call(kv(rows=0)) == skd.OK
    for call in (append, read):
        assert call(k=None) == call(v=None) == skd.ERR_NULL
        assert call(k=P + 2) == call(ks=504) == call(ks=516) == call(vs=0) == skd.ERR_SHAPE
    assert read(elem=2) == skd.ERR_SHAPE
    assert attend(q=None) == attend(o=None) == attend(k=P, ks=512) == attend(v=P, vs=512) == skd.ERR_NULL
    assert attend(qs=512) == attend(os_=1020) == attend(q=P + 8) == attend(heads=6) == attend(heads=0) == skd.ERR_SHAPE
    assert attend(k=P, ks=504, v=P, vs=512) == skd.ERR_SHAPE
    for s in (0.0, -1.0, float("nan"), float("inf")):
        assert attend(scale=s) == skd.ERR_RANGE
    # more workgroups than a launch has
    assert attend(kv(rows=1 << 30, max_pages=1 << 10)) == skd.ERR_RANGE
    assert append(kv(rows=1 << 30)) == read(kv(rows=1 << 30)) == skd.ERR_RANGE
    # a workspace is missing, too small, or not aligned
    long = dict(ch=chunk(max_past=100000), c=kv(max_pages=2000, rows=1))
    need = lib.skd_kv_attend_workspace(C.byref(long["c"]), C.byref(long["ch"]), 8)
    assert need > 0 and need % 4 == 0
    assert attend(**long) == skd.ERR_NULL and attend(**long, ws=P + 4, n=need) == skd.ERR_SHAPE and attend(**long, ws=P, n=need - 1) == skd.ERR_NOMEM


def test_draws():
    lib = skd.lib()

    need = lib.skd_sample_workspace(3, 1000)

    def rc(z=P, stride=1000, rows=3, vocab=1000, u=P, out=P, ws=P, n=1 << 30):
        return lib.skd_sample(z, stride, rows, vocab, None, u, out, ws, n, None)

    assert rc(z=None) == rc(u=None) == rc(out=None) == rc(ws=None) == skd.ERR_NULL
    assert rc(vocab=0) == rc(vocab=262145, stride=262145) == rc(stride=999) == rc(z=P + 2) == rc(out=P + 1) == rc(ws=P + 8) == skd.ERR_SHAPE
    assert need > 0 and rc(n=need - 1) == skd.ERR_NOMEM
    for name in ("temperature", "top_k", "top_p", "min_p"):
        bad = skd.Sampling(**{name: P + 2})
        assert lib.skd_sample(P, 1000, 3, 1000, C.byref(bad), P, P, P, need, None) == skd.ERR_SHAPE
    assert rc(rows=-1) == skd.ERR_RANGE and rc(rows=0) == skd.OK
    assert lib.skd_sample_workspace(-1, 10) == skd.ERR_RANGE and lib.skd_sample_workspace(1, 0) == lib.skd_sample_workspace(1, 1 << 19) == skd.ERR_SHAPE
    assert lib.skd_sample_workspace(128, 262144) >= 0
    assert lib.skd_logits_sample_rows(None, P, None, None, None) == skd.ERR_NULL

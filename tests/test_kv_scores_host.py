"""Refusals of the calls for changed scores, 4-bit pages and block tables, and places in a 4-bit page, on the CPU."""
import ctypes as C
import os
import subprocess

import pytest

from paper_2307_02628_amd import _build, skd
from test_kv_ops_host import P, attend, append, chunk, kv, read

KV4 = dict(elem=skd.KV_FP4)


@pytest.fixture(scope="module", autouse=True)
def _built():
    if not os.path.exists(skd.LIB_PATH):
        _build.build(force=True)


def scored(c=None, ch=None, sc=None, heads=8, scale=0.1, q=P, qs=1024, k=None, ks=0, v=None, vs=0, o=P, os_=1024, ws=None, n=0):
    return skd.lib().skd_kv_attend_scores(C.byref(c or kv()), C.byref(ch or chunk()), heads, scale, C.byref(sc or skd.Scores(cap=30.0)), q, qs, k, ks, v, vs, o, os_, ws, n, None)


def space(c=None, ch=None, sc=None, heads=8):
    return skd.lib().skd_kv_attend_scores_workspace(C.byref(c or kv()), C.byref(ch or chunk()), heads, C.byref(sc or skd.Scores()))


def test_pages_of_4_bits():
    lib = skd.lib()
    assert lib.skd_kv_page_bytes(C.byref(kv(**KV4))) == 4 * 2 * 34 * 128
    assert lib.skd_kv_page_bytes(C.byref(kv(**KV4, kv_heads=32, page_tokens=1 << 20, max_pages=1))) == 32 * (1 << 15) * 34 * 128
    for call in (append, read, attend, scored):
        assert call(kv(**KV4, pool=None)) == skd.ERR_NULL and call(kv(**KV4, pool=P + 8)) == skd.ERR_SHAPE
        assert call(kv(**KV4, rows=0)) == call(kv(**KV4), chunk(max_new=0)) == skd.OK
        assert call(kv(elem=3)) == call(kv(elem=5)) == call(kv(**KV4, head_dim=96)) == skd.ERR_SHAPE


def test_scores():
    lib = skd.lib()
    assert lib.skd_kv_attend_scores(C.byref(kv()), C.byref(chunk()), 8, 0.1, None, P, 1024, None, 0, None, 0, P, 1024, None, 0, None) == skd.ERR_NULL
    assert lib.skd_kv_attend_scores_workspace(C.byref(kv()), C.byref(chunk()), 8, None) == skd.ERR_NULL
    for bad in (-1.0, 1e-9, 1024.5, float("nan"), float("inf"), -float("inf")):
        assert scored(sc=skd.Scores(cap=bad)) == space(sc=skd.Scores(cap=bad)) == skd.ERR_RANGE
    assert scored(sc=skd.Scores(window=-1)) == space(sc=skd.Scores(window=-1)) == skd.ERR_RANGE
    assert scored(sc=skd.Scores(cap=2.0 ** -20), scale=1e37) == skd.ERR_RANGE           # 3 * scale / cap is no number
    for name in ("slopes", "begin", "end"):
        assert scored(sc=skd.Scores(**{name: P + 2})) == skd.ERR_SHAPE
    assert scored(q=None) == scored(o=None) == scored(k=P, ks=512) == scored(kv(pool=None)) == scored(None, chunk(first=None)) == skd.ERR_NULL
    assert scored(qs=512) == scored(os_=1020) == scored(q=P + 8) == scored(heads=6) == scored(heads=0) == skd.ERR_SHAPE
    for s in (0.0, -1.0, float("nan"), float("inf")):
        assert scored(scale=s) == skd.ERR_RANGE
    assert scored(None, chunk(max_new=0)) == scored(None, chunk(tokens=0)) == scored(kv(rows=0)) == skd.OK
    assert scored(kv(rows=1 << 30, max_pages=1 << 10)) == skd.ERR_RANGE


def test_workspace_of_windows():
    """A window bounds what there is to share out."""
    long = dict(ch=chunk(max_past=100000, max_new=1, tokens=1), c=kv(max_pages=2000, rows=1))
    need = space(**long)
    assert need > 0 and need == skd.lib().skd_kv_attend_workspace(C.byref(long["c"]), C.byref(long["ch"]), 8)
    assert scored(**long) == skd.ERR_NULL and scored(**long, ws=P + 4, n=need) == skd.ERR_SHAPE and scored(**long, ws=P, n=need - 1) == skd.ERR_NOMEM
    assert space(**long, sc=skd.Scores(window=64)) == 0 < space(**long, sc=skd.Scores(window=20000)) <= need
    assert space(**long, sc=skd.Scores(window=2 ** 31 - 1)) == need


def test_tables():
    lib = skd.lib()

    def assign(c=None, source=None, length=P, more=P, out=4 * P, copies=P, counts=P, ws=P, n=1 << 30):
        return lib.skd_kv_assign(C.byref(c or kv(pool=None)), source, length, more, out, copies, counts, ws, n, None)

    def compact(c=None, out=4 * P, copies=P, counts=P, ws=P, n=1 << 30):
        return lib.skd_kv_compact(C.byref(c or kv(pool=None)), out, copies, counts, ws, n, None)

    assert lib.skd_kv_assign_workspace(None) == lib.skd_kv_compact_workspace(None) == lib.skd_kv_copy_pages(None, P, 1, None, None) == skd.ERR_NULL
    assert assign(length=None) == assign(more=None) == skd.ERR_NULL
    for call in (assign, compact):
        assert call(out=None) == call(copies=None) == call(counts=None) == call(ws=None) == call(kv(block_table=None)) == skd.ERR_NULL
        assert call(out=4 * P + 1) == call(copies=P + 2) == call(counts=P + 3) == call(ws=P + 8) == call(kv(block_table=P + 2)) == skd.ERR_SHAPE
        assert call(out=P + 4) == call(out=P - 8) == skd.ERR_RANGE                        # overlaps the table
        assert call(n=0) == skd.ERR_NOMEM
        assert call(kv(rows=1 << 20, max_pages=1 << 11)) == call(kv(rows=1 << 25, max_pages=1)) == skd.ERR_RANGE
        assert call(kv(elem=9)) == call(kv(page_tokens=31)) == skd.ERR_SHAPE
    assert assign(source=P + 1) == assign(length=P + 1) == assign(more=P + 2) == skd.ERR_SHAPE
    assert assign(source=P, out=P) == skd.ERR_RANGE
    need = lib.skd_kv_assign_workspace(C.byref(kv()))
    assert need > 0 and assign(n=need - 1) == skd.ERR_NOMEM
    assert lib.skd_kv_assign_workspace(C.byref(kv(pages=2 ** 31 - 1))) > 4 * 4 * (2 ** 31 - 1)
    copy = lambda c=None, copies=P, most=3, number=None: lib.skd_kv_copy_pages(C.byref(c or kv()), copies, most, number, None)  # noqa: E731
    assert copy(most=-1) == skd.ERR_RANGE and copy(most=0) == skd.OK
    assert copy(copies=None) == copy(kv(pool=None)) == skd.ERR_NULL
    assert copy(copies=P + 2) == copy(number=P + 1) == copy(kv(pool=P + 4)) == skd.ERR_SHAPE


DRIVER = r"""
#include <cstdint>
#include <cstdio>
#include <vector>
#include <initializer_list>
#include "kv_pages.h"
using namespace skd;
#define EXPECT(c) do { if (!(c)) { printf("FAILED %s:%d: %s\n", __FILE__, __LINE__, #c); return 1; } } while (0)
int main() {
  // every byte of a page is one thing's: pairs of elements of a key or value, or an exponent
  for (int dh : {64, 128})
    for (int pt : {32, 96}) {
      const int H = 3;
      const KvGeom g{pt, 1, H, dh, 0};
      std::vector<int> hit(kv4_page_bytes(H, dh, pt), 0);
      auto mark = [&](long at) { return at >= 0 && at < (long)hit.size() && hit[at]++ == 0; };
      for (int h = 0; h < H; ++h)
        for (int t = 0; t < pt; ++t) {
          for (int e = 0; e < dh; e += 2) EXPECT(mark(kv4_k_off(h, t, e, g)));
          for (int i = 0; i < dh / 32; ++i) {
            for (int e = 0; e < 16; ++e) EXPECT(mark(kv4_v_off(h, t, 32 * i + e, g)));
            EXPECT(mark(kv4_k_exp_off(h, t, i, g)) && mark(kv4_v_exp_off(h, t, i, g)));
          }
        }
      for (int x : hit) EXPECT(x == 1);
    }
  // a page of more than 4 GiB: the parts of its last block lie behind each other
  const int pt = 1 << 20;
  const KvGeom g{pt, 1, 256, 128, 0};
  EXPECT(kv4_page_bytes(256, 128, pt) == 256L * (pt / 32) * 34 * 128);
  EXPECT(kv4_v_exp_off(255, pt - 1, 3, g) == kv4_page_bytes(256, 128, pt) - 1);
  EXPECT(kv4_k_off(255, pt - 32, 0, g) == kv4_page_bytes(256, 128, pt) - 34 * 128);
  printf("all checks passed\n");
  return 0;
}
"""


def test_places_of_4_bits(tmp_path):
    src = tmp_path / "driver.cpp"
    src.write_text(DRIVER)
    exe = str(tmp_path / "driver")
    subprocess.run(["g++", "-std=c++17", "-Wall", "-Werror", "-O2", "-fsanitize=undefined", "-I", _build.CSRC, str(src), "-o", exe], check=True)
    res = subprocess.run([exe], capture_output=True, text=True, timeout=60)
    assert res.returncode == 0 and "all checks passed" in res.stdout and not res.stderr, res.stdout + res.stderr

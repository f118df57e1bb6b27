"""kvr_rotate, kvr_attend_prompt and kvr_attend_paged without a GPU: what they refuse, and the arithmetic of pages, rows and
visible tiles that their kernels share, compiled for the host."""
import ctypes as C
import itertools
import os
import random
import subprocess

import pytest

from paper_2512_17917_amd import binding as kvr
from paper_2512_17917_amd import build as B

OK, E, U, W = kvr.KVR_OK, kvr.KVR_ERR_INVALID_ARG, kvr.KVR_ERR_UNSUPPORTED, kvr.KVR_ERR_WORKSPACE_TOO_SMALL
P, ODD = 0x10000, 0x10008                     # fake device addresses; never dereferenced


def _desc(batch=2, dtype=kvr.KVR_BF16):
    return kvr.make_desc(batch, 8, 2, 1, 1, dtype)


def _pages(**kw):
    a = dict(k=P, v=P, table=P, n_pages=10, page_size=16, table_cap=4)
    a.update(kw)
    return kvr.kvr_pages(*a.values())


def _rot(**kw):
    a = dict(q_weight=P, k_weight=P, inv_freq=P, eps=1e-6, rot_dim=128, style=0)
    a.update(kw)
    return kvr.kvr_rotation(*a.values())


def _rotate(desc=None, rot=None, pages=None, **kw):
    a = dict(q=P, q_stride=1536, k=P, k_stride=1536, v=P, v_stride=1536, n_rows=2, q_start=None, n_ctx=P, q_out=P + 16,
             k_out=P + 16)
    a.update(kw)
    d, r = desc or _desc(), rot or _rot()
    return kvr.lib().kvr_rotate(C.byref(d), C.byref(r), *a.values(), C.byref(pages) if pages else None, None)


def _prompt(desc=None, over=None, **kw):
    a = dict(q=P, n_rows=2, q_start=None, n_ctx=P, pages=C.byref(over or _pages()), window=0, n_sink=0, out=P + 16, scores=P,
             n_cap=64, ws=P, ws_bytes=0)             # too small a workspace: nothing is ever launched
    a.update(kw)
    return kvr.lib().kvr_attend_prompt(C.byref(desc or _desc()), *a.values(), None)


def _paged(desc=None, over=None, **kw):
    a = dict(q=P, n_ctx=P, pages=C.byref(over or _pages(table_cap=128)), window=0, n_sink=0, out=P + 16, scores=P, n_cap=64, ws=P, ws_bytes=0)
    a.update(kw)
    return kvr.lib().kvr_attend_paged(C.byref(desc or _desc()), *a.values(), None)


BAD_PAGES = [dict(k=None), dict(v=None), dict(k=ODD), dict(v=ODD), dict(table=P + 2), dict(n_pages=0), dict(n_pages=-1),
             dict(page_size=0), dict(page_size=(1 << 30) + 1), dict(table_cap=0), dict(page_size=1 << 20, table_cap=1025),
             dict(table=None, n_pages=1)]


@pytest.mark.parametrize("bad", BAD_PAGES)
def test_bad_pages_are_refused(bad):
    p = _pages(**bad)
    assert _rotate(pages=p, k_out=None) == E
    assert _prompt(over=p) == E
    assert _paged(over=p) == E


@pytest.mark.parametrize("bad", [dict(eps=-1.0), dict(eps=float("nan")), dict(eps=float("inf")), dict(rot_dim=-2), dict(rot_dim=3),
                                 dict(rot_dim=130), dict(style=2), dict(style=-1), dict(inv_freq=None), dict(inv_freq=P + 4),
                                 dict(q_weight=ODD), dict(k_weight=ODD)])
def test_bad_rotations_are_refused(bad):
    assert _rotate(rot=_rot(**bad)) == E


@pytest.mark.parametrize("bad", [dict(q=None), dict(q_out=None), dict(k=None), dict(k_out=None), dict(q=None, q_out=None, k=None, k_out=None),
                                 dict(n_ctx=None), dict(q=ODD), dict(k=ODD), dict(q_out=ODD), dict(k_out=ODD), dict(q_stride=1016),
                                 dict(q_stride=1028), dict(k_stride=255), dict(k_stride=260), dict(n_rows=-1), dict(n_rows=3),
                                 dict(n_rows=(1 << 27) + 1, q_start=P), dict(q_out=P), dict(k_out=P)])
def test_bad_rows_are_refused(bad):
    assert _rotate(**bad) == E


def test_rotate_with_pages_needs_values():
    p = _pages()
    for bad in (dict(v=None), dict(v=ODD), dict(v_stride=248), dict(v_stride=257), dict(k=None)):
        assert _rotate(pages=p, **bad) == E, bad


def test_no_rows_are_no_work():
    assert _rotate(n_rows=0, q_start=P, q=None, q_out=None, k=None, k_out=None) == OK
    assert _prompt(n_rows=0, q_start=P, q=None, out=None) == OK


@pytest.mark.parametrize("call", [_prompt, _paged])
def test_bad_attention_is_refused(call):
    assert call() == W                                    # as it should be but for the workspace
    for bad in (dict(q=None), dict(q=ODD), dict(n_ctx=None), dict(out=None), dict(out=ODD), dict(out=P), dict(pages=None), dict(window=-1),
                dict(n_sink=-1), dict(n_cap=0), dict(n_cap=(1 << 30) + 1), dict(ws=None), dict(ws=ODD)):
        assert call(**bad) == E, bad
    for field, value, code in (("head_dim", 64, U), ("n_q_heads", 6, U), ("batch", 0, E), ("dtype", 7, E)):
        d = _desc()
        setattr(d, field, value)
        assert call(desc=d) == code, field


def test_bad_prompt_rows_are_refused():
    assert _prompt(n_rows=-1) == E and _prompt(n_rows=3) == E and _prompt(n_rows=(1 << 27) + 1, q_start=P) == E


def test_workspace_sizes():
    L, d, n = kvr.lib(), _desc(), C.c_size_t(0)
    p = _pages(k=None, v=None)                            # the pools are not looked at

    def prompt(rows, scores, pages=p, window=0):
        assert L.kvr_attend_prompt_workspace_size(C.byref(d), rows, C.byref(pages), window, 0, scores, C.byref(n)) == OK
        return n.value

    def paged(scores, pages=p):
        assert L.kvr_attend_paged_workspace_size(C.byref(d), C.byref(pages), 0, 0, scores, C.byref(n)) == OK
        return n.value
    assert prompt(0, 1) == 0
    assert prompt(100, 1) >= 100 * 8 * 4                  # a float per row and head
    assert paged(1) == paged(0) == 0                      # 64 tokens: a workgroup has all of a head's
    big = _pages(k=None, v=None, table_cap=8192)
    assert paged(1, big) >= paged(1) and paged(1, big) >= paged(0, big)
    for f, args in ((L.kvr_attend_prompt_workspace_size, (5,)), (L.kvr_attend_paged_workspace_size, ())):
        assert f(C.byref(d), *args, C.byref(p), 0, 0, 0, None) == E
        assert f(C.byref(d), *args, None, 0, 0, 0, C.byref(n)) == E
        assert f(C.byref(d), *args, C.byref(p), -1, 0, 0, C.byref(n)) == E
        assert f(None, *args, C.byref(p), 0, 0, 0, C.byref(n)) == E
        assert f(C.byref(d), *args, C.byref(_pages(page_size=0)), 0, 0, 0, C.byref(n)) == E
    assert L.kvr_attend_prompt_workspace_size(C.byref(d), -1, C.byref(p), 0, 0, 0, C.byref(n)) == E


def test_more_tokens_than_the_chunks_numbers_hold_are_refused():
    """2^37 tokens of cache (a table that names the same pages again and again)."""
    d = kvr.make_desc(4096, 8, 8, 1, 1, kvr.KVR_BF16)
    big, less = _pages(page_size=1024, table_cap=4096), _pages(page_size=1024, table_cap=4095)
    n = C.c_size_t(0)
    for p, want in ((big, U), (less, OK)):
        assert kvr.lib().kvr_attend_paged_workspace_size(C.byref(d), C.byref(p), 0, 0, 0, C.byref(n)) == want
    assert _paged(desc=d, over=big, n_cap=64) == U and _paged(desc=d, over=less) == W
    assert _paged(desc=d, over=big, window=5000) == W
    rows = dict(n_rows=5, q_start=P)
    assert _prompt(desc=d, over=big, **rows) == U and _prompt(desc=d, over=less, **rows) == W


def test_binding_refuses_what_does_not_fit():
    import torch
    d = _desc()
    x = torch.zeros(4, 2, 16, 128, dtype=torch.bfloat16)
    with pytest.raises(ValueError):
        kvr.make_pages(d, x, x)                           # host memory
    with pytest.raises(ValueError):
        kvr.make_pages(d, x[:, :1], x)                    # heads
    with pytest.raises(ValueError):
        kvr.make_pages(d, x[0], x[0])
    with pytest.raises(ValueError):
        kvr.make_rotation(d, torch.zeros(64, dtype=torch.float64))
    with pytest.raises(TypeError):
        kvr.kvr_attend_paged(d, x, x, None, 0, 0, x, None, 0, None)
    with pytest.raises(TypeError):
        kvr.kvr_rotate(d, None, x, x, x, 2, None, x, x)


# ---------------------------------------------------------------------------
PROBE = r"""
#include <cstdio>
#include <vector>
#include "kvr_pages.h"
// r page_size j -> quotient | t window n_sink lo hi -> tiles of 16: ahead start n | a n_pages page heads b h j entry -> row |
// s n_rows first next -> row span
int main() {
  char kind;
  while (std::scanf(" %c", &kind) == 1) {
    if (kind == 'r') {
      kvr_pages c = {};
      int j;
      if (std::scanf("%d %d", &c.page_size, &j) != 2) return 1;
      std::printf("%d\n", kvr::page_index(kvr::dev_pages(c), j));
    } else if (kind == 't') {
      kvr::Visible v;
      int lo, hi;
      if (std::scanf("%d %d %d %d", &v.window, &v.n_sink, &lo, &hi) != 4) return 1;
      const kvr::TileRange r = kvr::tile_range<16>(v, lo, hi);
      for (int i = 0; i < r.n; ++i) std::printf("%d ", kvr::tile_token<16>(r, i));
      std::printf("\n");
    } else if (kind == 'a') {
      kvr_pages c = {};
      int heads, b, h, j, entry;
      if (std::scanf("%d %d %d %d %d %d %d", &c.n_pages, &c.page_size, &heads, &b, &h, &j, &entry) != 7) return 1;
      c.table_cap = j / c.page_size + 1;
      std::vector<int32_t> table((size_t)(b + 1) * c.table_cap, 0);
      table[(size_t)b * c.table_cap + j / c.page_size] = entry;
      c.table = table.data();
      std::printf("%lld\n", kvr::page_row(kvr::dev_pages(c), heads, b, h, j));
    } else if (kind == 's') {
      int n_rows, q[2];
      if (std::scanf("%d %d %d", &n_rows, &q[0], &q[1]) != 3) return 1;
      const kvr::RowSpan s = kvr::row_span(q, n_rows, 0);
      std::printf("%d %d\n", s.first, s.n);
    }
  }
}
"""


@pytest.fixture(scope="module")
def ask(tmp_path_factory):
    d = tmp_path_factory.mktemp("pages")
    src, exe = str(d / "probe.hip"), str(d / "probe")
    open(src, "w").write(PROBE)
    subprocess.run([B._hipcc(), "--offload-host-only", "-std=c++17", "-I", B.CSRC, src, "-o", exe], check=True, capture_output=True)

    def run(lines):
        out = subprocess.run([exe], input="\n".join(lines) + "\n", capture_output=True, text=True, check=True).stdout
        return [tuple(map(int, x.split())) for x in out.splitlines()]
    return run


def test_page_of_a_token(ask):
    """The quotient by product, at the borders of pages of every kind of size, up to the last token there can be."""
    top = (1 << 30) - 1
    sizes = [1, 2, 3, 5, 7, 15, 16, 17, 24, 48, 63, 64, 65, 100, 127, 128, 255, 256, 1000, 4095, 4096, 65537, 10 ** 6 + 3,
             (1 << 29) - 1, 1 << 29, top, 1 << 30]
    rng = random.Random(3)
    cases = [(s, j) for s in sizes for k in [0, 1, 2, 3, top // s - 1, top // s] + [rng.randint(0, top // s) for _ in range(50)]
             for j in (k * s - 1, k * s, k * s + 1) if 0 <= j <= top]
    got = ask([f"r {s} {j}" for s, j in cases])
    assert [g[0] for g in got] == [j // s for s, j in cases]


def test_row_of_a_token_and_pages_that_are_not_there(ask):
    cases = []
    for ps in (1, 16, 24, 1000):
        for entry in (0, 1, 9, 10, 11, -1, -2 ** 31, 2 ** 31 - 1):
            cases.append((10, ps, 8, 2, 5, 3 * ps + ps // 2, entry))
    cases.append((2 ** 21, 1024, 8, 0, 7, 1023, 2 ** 21 - 1))       # past 2^32 rows, as 64-bit numbers
    got = ask(["a " + " ".join(map(str, c)) for c in cases])
    for (n_pages, ps, heads, b, h, j, entry), (row,) in zip(cases, got):
        assert row == ((entry * heads + h) * ps + j % ps if 0 <= entry < n_pages else -1)


def test_tiles_hold_what_queries_see_once(ask):
    """Every token that a query at lo .. hi sees lies in exactly one tile, tiles do not overlap, and none lies wholly
    beyond what any of them sees."""
    cases = [(w, s, lo, lo + more) for w, s, lo, more in itertools.product(
        (0, 1, 2, 15, 16, 17, 40, 100, 1 << 30), (0, 1, 4, 15, 16, 17, 33, 64, 200, 1 << 30), (-5, -1, 0, 1, 14, 15, 16, 31, 47, 48, 100),
        (0, 1, 7, 15, 16, 33))]
    got = ask([f"t {w} {s} {lo} {hi}" for w, s, lo, hi in cases])
    for (w, s, lo, hi), tiles in zip(cases, got):
        seen = {j for p in range(max(lo, 0), hi + 1) for j in range(p + 1) if w == 0 or j > p - w or j < s}
        assert len(set(tiles)) == len(tiles) and all(t % 16 == 0 and t >= 0 for t in tiles), (w, s, lo, hi)
        held = {t + i for t in tiles for i in range(16)}
        assert seen <= held, (w, s, lo, hi)
        reach = {j for p in range(lo, hi + 1) for j in range(p + 1) if w == 0 or j > p - w or j < s}
        assert all(any(t + i in reach for i in range(16)) for t in tiles), (w, s, lo, hi)


def test_row_spans_are_clamped(ask):
    cases = [(10, 0, 3), (10, 3, 3), (10, -4, 2), (10, 8, 30), (10, 30, 40), (10, 7, 2), (10, -5, -1)]
    want = [(0, 3), (3, 0), (0, 2), (8, 2), (10, 0), (7, 0), (0, 0)]
    assert ask(["s " + " ".join(map(str, c)) for c in cases]) == want

"""kvr_attend_shared without a GPU: what it, make_groups and PagedCache refuse, the C route beside the Python checks, and how its work
is cut, compiled for the host."""
import ctypes as C
import os
import random
import subprocess

import pytest
import torch

from paper_2512_17917_amd import binding as kvr
from paper_2512_17917_amd import build as B
from paper_2512_17917_amd.state import LayerState, PagedCache
from tests.test_cache_binding_cpu import _cache_of
from tests.test_cache_fast_cpu import Fake, _both, _desc as _fake_desc, _pages as _fake_pages, _plain
from tests.test_cache_ops_cpu import BAD_PAGES, E, ODD, OK, P, U, W, _desc, _pages


def _groups(start=P, n_shared=P, n_groups=1):
    return kvr.kvr_groups(start, n_shared, n_groups)


def _shared(desc=None, over=None, groups=None, no_groups=False, **kw):
    a = dict(q=P, n_rows=2, q_start=None, n_ctx=P, pages=C.byref(over or _pages(table_cap=1 << 20)),
             groups=None if no_groups else C.byref(groups or _groups()), window=0, n_sink=0, out=P + 16, scores=P, n_cap=64, ws=P, ws_bytes=0)
    a.update(kw)                                     # too small a workspace: nothing is ever launched
    return kvr.lib().kvr_attend_shared(C.byref(desc or _desc()), *a.values(), None)


def _size(desc=None, n_rows=2, pages=None, groups=None, window=0, n_sink=0, scores=1, no_groups=False):
    n = C.c_size_t(0)
    rc = kvr.lib().kvr_attend_shared_workspace_size(C.byref(desc or _desc()), n_rows, C.byref(pages or _pages(table_cap=1 << 20)),
                                                    None if no_groups else C.byref(groups or _groups()), window, n_sink, scores, C.byref(n))
    return rc, n.value


@pytest.mark.parametrize("rows", [dict(), dict(q_start=P), dict(q_start=P, n_rows=7)])
def test_bad_attention_is_refused(rows):
    assert _shared(**rows) == W                           # as it should be but for the workspace
    for bad in (dict(q=None), dict(q=ODD), dict(n_ctx=None), dict(out=None), dict(out=ODD), dict(out=P), dict(pages=None), dict(window=-1),
                dict(n_sink=-1), dict(n_cap=0), dict(n_cap=(1 << 30) + 1), dict(ws=None), dict(ws=ODD), dict(n_rows=-1)):
        assert _shared(**{**rows, **bad}) == E, bad
    for field, value, code in (("head_dim", 64, U), ("n_q_heads", 6, U), ("batch", 0, E), ("dtype", 7, E)):
        d = _desc()
        setattr(d, field, value)
        assert _shared(desc=d, **rows) == code, field


@pytest.mark.parametrize("bad", [dict(n_groups=-1), dict(n_groups=3), dict(start=None), dict(n_shared=None), dict(start=P + 2),
                                 dict(n_shared=P + 1)])
def test_bad_groups_are_refused(bad):
    g = _groups(**bad)
    assert _shared(groups=g) == E and _shared(groups=g, q_start=P) == E
    assert _size(groups=g)[0] == (E if "n_groups" in bad else OK)            # (which looks at their number alone)


@pytest.mark.parametrize("bad", BAD_PAGES)
def test_bad_pages_are_refused(bad):
    assert _shared(over=_pages(**bad)) == E


def test_rows_that_are_not_the_sequences():
    assert _shared(n_rows=3) == E and _shared(n_rows=1) == E
    few = _pages()                                               # (64 tokens)
    for n, code in ((1 << 22, W), ((1 << 22) + 1, E)):           # times 8 heads: 2^25, which the join's launch has place for
        assert _shared(n_rows=n, q_start=P, over=few) == code
        assert _size(n_rows=n, pages=few)[0] == (OK if code == W else E)
    assert _size(n_rows=-1)[0] == E


def test_no_rows_and_no_groups():
    assert _shared(n_rows=0, q_start=P, q=None, out=None) == OK
    assert _size(n_rows=0) == (OK, 0)
    for kw in (dict(no_groups=True), dict(groups=_groups(None, None, 0))):
        assert _shared(**kw) == W and _shared(q_start=P, **kw) == W


def test_work_past_31_bits_is_refused():
    """2 (ceil(n_rows G / 16) + B) Hkv (7 (tiles of 64 tokens + 2) + 12), and the pages' own bound."""
    d = kvr.make_desc(2, 8, 2, 1, 1, kvr.KVR_BF16)
    row = lambda n_rows, cap: 2 * (-(-n_rows * 4 // 16) + 2) * 2 * (7 * (-(-cap // 64) + 2) + 12)
    cap = 1 << 29
    pages = _pages(page_size=1024, table_cap=cap // 1024)
    n = max(x for x in range(1, 200) if row(x, cap) < 2 ** 31 - 1)
    assert n < 199
    assert _size(n_rows=n, pages=pages)[0] == OK and _size(n_rows=n + 1, pages=pages)[0] == U
    assert _shared(n_rows=n, q_start=P, over=pages) == W and _shared(n_rows=n + 1, q_start=P, over=pages) == U
    d = kvr.make_desc(4096, 8, 8, 1, 1, kvr.KVR_BF16)
    big = _pages(page_size=1024, table_cap=4096)
    assert _size(desc=d, n_rows=4096, pages=big)[0] == U


def test_a_workspace_of_the_size_given_is_enough():
    """For one row a sequence the size is asked for without saying whether there will be starts; with fewer scores than tokens
    less is needed."""
    for dtype in (kvr.KVR_BF16, kvr.KVR_F32):
        for batch in (1, 2, 40, 700):
            d = kvr.make_desc(batch, 8, 2, 1, 1, dtype)
            for cap in (1, 3, 30, 200, 1000, 1 << 15):
                pages = _pages(table_cap=cap)
                for rows in (1, batch, 3 * batch + 1):
                    for window, scores, g in ((0, 0, 0), (0, 1, 1), (900, 1, 1), (900, 0, 1), (0, 1, 0)):
                        kw = dict(groups=_groups(n_groups=g))
                        rc, n = _size(d, rows, pages, window=window, scores=scores, **kw)
                        assert rc == OK
                        if n == 0:
                            continue
                        for n_cap in (1, 70, 16 * cap) if scores else (0,):
                            for q_start in (P, None) if rows == batch else (P,):
                                need = _least(d, rows, pages, q_start, window, scores, n_cap, kw["groups"], n)
                                assert need <= n


def _least(d, rows, pages, q_start, window, scores, n_cap, groups, most):
    """The smallest workspace that is not refused, found without a launch: one that is large enough but not aligned is
    refused as such."""
    call = lambda n: _shared(d, pages, groups, n_rows=rows, q_start=q_start, window=window, scores=P if scores else None, n_cap=n_cap,
                             ws=P + 8, ws_bytes=n)
    return most if call(most) == E else most + 1


def test_make_groups():
    i32 = lambda n, at=0x1000, **kw: Fake(torch.int32, (n,), at, **kw)
    for start, n in ((None, i32(1)), (i32(2), None), ([0, 1], [5]), (i32(1), i32(1)), (i32(2), Fake(torch.int64, (1,), 0x1000)),
                     (i32(2, cuda=False), i32(1)), (i32(2), i32(1, dev=1)), (i32(2, strides=(2,)), i32(1))):
        with pytest.raises((ValueError, TypeError)):
            kvr.make_groups(start, n)
    g = kvr.make_groups(i32(4), i32(3, 0x2000))
    assert (g.start, g.n_shared, g.n_groups) == (0x1000, 0x2000, 3)


# ---------------------------------------------------------------------------
@pytest.fixture()
def fast(monkeypatch):
    if not os.path.exists(B.FAST):
        pytest.skip("the extension was left out of the build")
    real, got = kvr.lib(), []
    m = kvr._fast
    I, L, V = C.c_int32, C.c_int64, C.c_void_p
    fn = C.CFUNCTYPE(I, V, V, I, V, V, V, V, I, I, V, V, L, V, C.c_size_t, V)(lambda *a: got.append(a) or 0)
    at = lambda f: C.cast(f, V).value
    m.setup_more(at(real.kvr_rotate_axes), at(fn))

    class Recorder:
        kvr_attend_shared = staticmethod(lambda *a: got.append(tuple(_plain(x) for x in a)) or 0)

    monkeypatch.setattr(kvr, "lib", lambda: Recorder)
    monkeypatch.setattr(kvr, "_stream", lambda: 77)
    monkeypatch.setattr(kvr, "_stream_of", lambda dev: 77)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    yield got
    m.setup_more(at(real.kvr_rotate_axes), at(real.kvr_attend_shared))


def _args(**kw):
    bf, i32 = torch.bfloat16, torch.int32
    a = dict(q=Fake(bf, (5, 8, 128), 0x1000), n_rows=5, q_start=Fake(i32, (4,), 0x4000), n_ctx=Fake(i32, (3,), 0x5000), pages=None, groups=None,
             window=5, n_sink=2, out=Fake(bf, (5, 8, 128), 0x6000), scores=Fake(torch.float32, (3, 2, 40), 0x7000), n_cap=40,
             ws=Fake(torch.uint8, (999,), 0x8000))
    a.update(kw)
    return a


def _call(d, **kw):
    a = _args(**kw)
    a["pages"] = _fake_pages(d)
    kvr.kvr_attend_shared(d, *a.values())


def _some_groups(dev=0):
    return kvr.make_groups(Fake(torch.int32, (3,), 0x21000, dev=dev), Fake(torch.int32, (2,), 0x22000, dev=dev))


CALLS = [dict(), dict(scores=None, n_cap=0), dict(ws=None), dict(n_rows=0), dict(n_rows=3, q_start=None)]


@pytest.mark.parametrize("case", range(len(CALLS)))
@pytest.mark.parametrize("grouped", [False, True])
def test_both_routes_pass_the_same(fast, monkeypatch, case, grouped):
    d = _fake_desc()
    g = _some_groups() if grouped else None
    pages = _fake_pages(d)
    a = _args(**CALLS[case])
    a.update(pages=pages, groups=g)
    one, two = _both(monkeypatch, lambda: kvr.kvr_attend_shared(d, *a.values()), fast)
    assert one == two


BAD = [dict(q=Fake(torch.float32, (5, 8, 128), 0x1000)), dict(q=Fake(torch.bfloat16, (4, 8, 128), 0x1000)), dict(q_start=Fake(torch.int32, (3,), 0x4000)),
       dict(n_ctx=Fake(torch.int32, (2,), 0x5000)), dict(n_ctx=None), dict(out=Fake(torch.bfloat16, (5, 8, 127), 0x6000)),
       dict(scores=Fake(torch.float32, (3, 2, 39), 0x7000)), dict(out=Fake(torch.bfloat16, (5, 8, 128), 0x6000, dev=1)),
       dict(n_ctx=Fake(torch.int32, (3,), 0x5000, cuda=False)), dict(ws=Fake(torch.uint8, (999,), 0x8000, dev=1))]


@pytest.mark.parametrize("case", range(len(BAD)))
@pytest.mark.parametrize("route", ["C", "Python"])
def test_bad_tensors_are_refused(fast, monkeypatch, case, route):
    if route == "Python":
        monkeypatch.setattr(kvr, "_fast", None)
    with pytest.raises((ValueError, TypeError)):
        _call(_fake_desc(), groups=_some_groups(), **BAD[case])
    assert not fast


def test_groups_of_another_device_or_none_made_are_refused(fast):
    for g in (_some_groups(dev=1), kvr.kvr_groups(), (1, 2)):
        with pytest.raises((ValueError, TypeError)):
            kvr.kvr_attend_shared(_fake_desc(), *{**_args(), "pages": _fake_pages(_fake_desc()), "groups": g}.values())
    assert not fast


# ---------------------------------------------------------------------------
def _cache(n_pages=9, page=4, cols=4):
    c = _cache_of([[-1] * cols, [-1] * cols, [-1] * cols], [0, 0, 0], n_pages, page)
    c.device, c.n_cap = torch.device("cpu"), page * cols
    c.scores = torch.rand(3, 2, page * cols)
    return c


@pytest.mark.parametrize("n", [0, 1, 4, 7, 8, 15, 16])
def test_a_sequence_begins_with_anothers_tokens(n):
    c = _cache()
    c.assign(0, 0, [5, 2, 8, 0])
    c.assign(1, 0, [3, 3, 3, 3])
    k, v, sc = c.k.clone(), c.v.clone(), c.scores.clone()
    c.begin_with(1, 0, n, page=7)
    full, rest = divmod(n, 4)
    assert c.table[1].tolist() == ([5, 2, 8, 0][:full] + [7] * (rest > 0) + [-1] * 4)[:4]
    assert c.table[0].tolist() == [5, 2, 8, 0] and c.table[2].tolist() == [-1] * 4
    for now, was in ((c.k, k), (c.v, v)):
        if rest:
            was[7, :, :rest] = was[[5, 2, 8, 0][full], :, :rest]
        assert torch.equal(now, was)
    sc[1, :, :n], sc[1, :, n:] = sc[0, :, :n], 0
    assert torch.equal(c.scores, sc)
    again = c.table.clone()
    c.begin_with(1, 0, n, page=7)                                # as another layer that shares the table does
    assert torch.equal(c.table, again)


def test_tokens_on_no_page_are_on_none_for_who_begins_with_them():
    for entry in (-1, 9, -2 ** 31):
        c = _cache()
        c.assign(0, 0, [5, entry])
        c.begin_with(1, 0, 6, page=7)
        assert c.table[1].tolist() == [5, -1, -1, -1]


@pytest.mark.parametrize("bad", [(0, 0, 4), (3, 0, 4), (0, 3, 4), (-1, 0, 4), (0, -1, 4), (1, 0, -1), (1, 0, 17), (1, 0, 5), (1, 0, 5, 9),
                                 (1, 0, 5, -1)])
def test_beginnings_that_cannot_be_are_refused(bad):
    c = _cache()
    before = c.table.clone()
    with pytest.raises(ValueError):
        c.begin_with(*bad)
    assert torch.equal(c.table, before)


def test_axes_and_positions_come_together():
    d = kvr.make_desc(2, 8, 2, 3, 5, torch.bfloat16, seed=1)
    s = LayerState.__new__(LayerState)
    s.desc, s.k_turned, s.q_turned, s.n_ctx = d, 0, 0, None
    for kw in (dict(axes=kvr.make_axes([0] * 64)), dict(pos=torch.zeros(1, 2, dtype=torch.int32))):
        with pytest.raises(ValueError):
            s.rotate(torch.zeros(2, 2, 128), torch.zeros(2, 8, 128), kvr.make_rotation(d), **kw)
    c = PagedCache.__new__(PagedCache)
    c.desc, c.rotation, c.n_ctx, c.q, c.pages, c.groups = d, None, torch.zeros(2), None, None, None
    for axes, pos in ((kvr.make_axes([0] * 64), None), (None, torch.zeros(1, 2, dtype=torch.int32))):
        c.axes = axes
        with pytest.raises(ValueError):
            c.decode_step(None, None, None, bump_n_ctx=False, pos=pos)


# ---------------------------------------------------------------------------
PROBE = r"""
#include <cstdio>
#include <vector>
#include "kvr_shared.h"
// One batch: which row, workgroups, B G Hkv n_rows cap window n_sink n_groups, own tokens that the join takes, then n_ctx, whether there are starts and they, groups' starts, tokens in
// common -> a line a piece: workgroup, of a sequence, its or the group's number, tile of columns, head, columns' place, columns, bits, from, lim, run, i0, i1
using namespace kvr;
template <typename Row, int COLS>
void pieces(const DevDesc& d, const SharedArgs& s, int wgs) {
  std::vector<typename Row::Entry> row;
  for (int g = 0; g < s.n_groups; ++g) row.push_back(Row::group_entry(d, s, g));
  for (int b = 0; b < d.B; ++b) {
    int common = 0;
    for (int g = 0; g < s.n_groups; ++g) {
      const Group x = group_at(s, d.B, g);
      if (b >= x.b0 && b < x.b1) common = x.common;
    }
    row.push_back(Row::member_entry(d, s, b, member_at(s, b, common)));
  }
  long long all = 0;
  int least = Row::LIGHT;
  for (auto& e : row) {
    all += (long long)Row::unit_length(e) * e.units;
    if (e.units > 0 && e.weight > Row::LIGHT) least = Row::HEAVY;
  }
  std::printf("%lld\n", all);
  const long long even = (all + wgs - 1) / wgs, per = even > least ? even : least;
  for (int w = 0; w * per < all; ++w) {
    const int at = (int)(w * per), end = (int)(at + per < all ? at + per : all);
    long long first = 0;
    for (auto& e : row)
      for (int u = 0; u < e.units; ++u, first += Row::unit_length(e)) {
        if (first + Row::unit_length(e) <= at || first >= end) continue;
        const Piece p = Row::piece_of(d, e, u, (int)first, at, end);
        const int some = p.cols - p.ct * COLS < COLS ? p.cols - p.ct * COLS : COLS;
        std::printf("%d %d %d %d %d %d %d %d %d %d %d %d %d %d %d %d %d\n", w, e.own, e.id, p.ct, p.h,
                    Row::place(d, s.a.n_rows, e.own, p.row0, p.cols, p.ct, p.h), some, p.bits, p.from, p.lim, p.ahead0, p.ahead, p.start, e.run.n, p.i0, p.i1, p.b);
      }
  }
  std::printf("end\n");
}
int main() {
  int which, wgs, starts;
  while (std::scanf("%d %d", &which, &wgs) == 2) {
    DevDesc d = {};
    SharedArgs s = {};
    if (std::scanf("%d %d %d %d %d %d %d %d %d", &d.B, &d.G, &d.Hkv, &s.a.n_rows, &s.a.pages.cap, &s.a.vis.window, &s.a.vis.n_sink, &s.n_groups, &s.own_most) != 9) return 1;
    d.Hq = d.G * d.Hkv;
    auto list = [](int n) {
      std::vector<int32_t> x(n + 1);
      for (int i = 0; i < n; ++i)
        if (std::scanf("%d", &x[i]) != 1) x[i] = 0;
      return x;
    };
    const std::vector<int32_t> n_ctx = list(d.B);
    if (std::scanf("%d", &starts) != 1) return 1;
    const std::vector<int32_t> q_start = list(starts ? d.B + 1 : 0), start = list(s.n_groups + 1), common = list(s.n_groups);
    s.a.n_ctx = n_ctx.data();
    s.a.q_start = starts ? q_start.data() : nullptr;
    s.start = start.data();
    s.n_shared = common.data();
    if (which == 0) pieces<WorkRow<256, 64>, 256>(d, s, wgs);
    else if (which == 1) pieces<WorkRow<16, 64>, 16>(d, s, wgs);
    else pieces<WorkRow<64, 64, true>, 64>(d, s, wgs);
  }
}
"""


@pytest.fixture(scope="module")
def ask(tmp_path_factory):
    d = tmp_path_factory.mktemp("shared")
    src, exe = str(d / "probe.hip"), str(d / "probe")
    open(src, "w").write(PROBE)
    subprocess.run([B._hipcc(), "--offload-host-only", "-std=c++17", "-I", B.CSRC, src, "-o", exe], check=True, capture_output=True)
    return lambda line: subprocess.run([exe], input=line + "\n", capture_output=True, text=True, check=True).stdout.splitlines()


def _batches():
    rng = random.Random(7)
    out = []
    for i in range(120):
        B, G, Hkv = rng.choice([1, 2, 5, 40, 90]), rng.choice([1, 2, 4, 8]), rng.choice([1, 2, 3])
        cap = rng.choice([1, 64, 500, 3000])
        starts = rng.random() < 0.5
        y = [rng.choice([0, 1, 1, 2, 5, 40]) if starts else 1 for _ in range(B)]
        q_start = [rng.choice([0, 3])]
        for n in y:
            q_start.append(q_start[-1] + n)
        n_rows = q_start[-1] + rng.choice([0, 2]) if starts else B
        cuts = sorted(rng.sample(range(B + 1), min(rng.randint(0, 6), B) + 1)) if rng.random() < 0.9 else list(range(B + 1))
        common = [rng.choice([0, 1, 63, 64, 65, 200, 450, 2900, 5000]) for _ in cuts[1:]]
        n = [rng.choice([0, 1, cap, rng.randint(0, cap + 10)]) for _ in range(B)]
        for (lo, hi), c in zip(zip(cuts, cuts[1:]), common):
            for b in range(lo, hi):
                if rng.random() < 0.8:
                    n[b] = c + y[b] + rng.randint(0, 90)
        window, sink = rng.choice([(0, 0), (0, 9), (1, 0), (70, 4), (64, 130), (500, 64)])
        out.append((B, G, Hkv, n_rows, cap, window, sink, n, q_start if starts else None, cuts, common, y))
    return out


@pytest.mark.parametrize("most_own", [0, 256])
@pytest.mark.parametrize("which,cols,wgs", [(0, 256, 256), (1, 16, 512), (2, 64, 512), (0, 256, 3), (1, 16, 1)])
def test_every_tile_of_every_unit_is_taken_once(ask, which, cols, wgs, most_own):
    for B, G, Hkv, n_rows, cap, window, sink, n, q_start, cuts, common, y in _batches():
        if most_own and q_start is not None:
            continue                                             # (one new row a sequence alone)
        words = [which, wgs, B, G, Hkv, n_rows, cap, window, sink, len(common), most_own, *n, int(q_start is not None), *(q_start or []), *cuts, *common]
        lines = ask(" ".join(map(str, words)))
        assert lines[-1] == "end"
        length = int(lines[0])
        most = 2 * (-(-n_rows * G // 16) + B) * Hkv * (7 * (-(-cap // 64) + 2) + 12)      # what the host allows for
        assert length <= most
        pieces = [tuple(map(int, x.split())) for x in lines[1:-1]]
        units, places = {}, {}
        for w, own, i, ct, h, c0, some, bits, lo, lim, ahead0, ahead, start, tiles, i0, i1, b in pieces:
            assert 0 <= i0 <= i1 <= tiles and 0 <= b < B and w < wgs
            u = units.setdefault((own, i, ct, h), dict(taken=[], first=[], last=[], lo=lo, lim=lim, tiles=tiles, run=(ahead0, ahead, start)))
            if i0 == i1:
                continue
            u["taken"] += range(i0, i1)
            u["first"] += [w] if bits & 2 and i0 == 0 else []
            u["last"] += [w] if bits & 4 and i1 == tiles else []
            u.setdefault("wgs", []).append(w)
            assert c0 >= 0 and c0 + some <= 2 * n_rows * G * Hkv
            for c in range(c0, c0 + some):                       # nobody else's place
                assert places.setdefault(cols * w + c, (own, i, ct, h, w)) == (own, i, ct, h, w)
        for key, u in units.items():
            assert sorted(u["taken"]) == list(range(u["tiles"])), key
            assert len(u["first"]) == len(u["last"]) == 1, key
            if which < 2:                                        # (the scores' pass leaves no pieces to join)
                assert sorted(set(u["wgs"])) == list(range(u["first"][0], u["last"][0] + 1)), key
        # what each row's columns see lies in its units' tiles
        cap_of = lambda x: min(max(x, 0), cap)
        group = {b: g for g, (lo, hi) in enumerate(zip(cuts, cuts[1:])) for b in range(lo, hi)}
        for b in range(B):
            m = cap_of(n[b])
            for t in {0, y[b] - 1} if y[b] else ():
                pos = m - y[b] + t
                seen = {j for j in range(pos + 1) if window == 0 or j > pos - window or j < sink}
                held = []
                for (own, i, ct, h), u in units.items():
                    if h or ct or (i != b if own else group.get(b) != i):
                        continue
                    if not own and m - y[b] < u["lim"]:
                        continue                                # a row among what is shared: by itself
                    ahead0, ahead, start = u["run"]
                    for k in range(u["tiles"]):
                        at = ahead0 + 64 * k if k < ahead else start + 64 * (k - ahead)
                        held += range(max(at, u["lo"]), min(at + 64, u["lim"]))
                if most_own and (1, b, 0, 0) not in units:       # the join's: its last tokens, no more than it takes
                    left = seen - set(held)
                    assert not left or m - min(left) <= most_own
                    assert not left or not held or max(held) < min(left)
                    held += left
                assert len(held) == len(set(held)) and seen <= set(held), (b, t)

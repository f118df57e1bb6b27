"""kvr_rotate, kvr_attend_prompt and kvr_attend_paged against float64 (tests/cache_ref.py)."""
import math

import pytest
import torch

from paper_2512_17917_amd import binding as kvr
from tests import cache_ref as R

pytestmark = [pytest.mark.gpu, pytest.mark.timeout(300)]
D = 128
BF, F32 = torch.bfloat16, torch.float32


def _normal(g, *shape, dtype):
    return torch.randn(shape, generator=g).to(dtype)


def _cache(g, B, Hkv, cap, page, dtype, *, spare=3):
    """Pools on the CPU and a table in no order (page 0: dense, no table)."""
    if page == 0:
        return _normal(g, B, Hkv, cap, D, dtype=dtype), _normal(g, B, Hkv, cap, D, dtype=dtype), None
    each = -(-cap // page)
    n = B * each + spare
    table = torch.randperm(n, generator=g)[:B * each].to(torch.int32).view(B, each)
    return _normal(g, n, Hkv, page, D, dtype=dtype), _normal(g, n, Hkv, page, D, dtype=dtype), table


def _starts(news, lead=0):
    out = [lead]
    for y in news:
        out.append(out[-1] + y)
    return out


def _dev(*ts):
    return [t.cuda() if t is not None else None for t in ts]


# ---------------------------------------------------------------------------
ROTATE = [  # dtype, heads, rot, pairs, norm, page, lengths, new (None: one row per sequence), first row
    (BF, (32, 8), 128, False, True, 0, [32768], None, 0),
    (BF, (32, 8), 128, False, True, 16, [1, 1000, 1048576 // 16], None, 0),
    (BF, (8, 2), 128, False, True, 64, [200, 0, 77], [200, 0, 5], 0),
    (BF, (8, 8), 64, True, True, 24, [31, 1, 130], [31, 1, 100], 3),
    (BF, (64, 8), 32, False, False, 100, [129], [129], 0),
    (BF, (3, 3), 20, False, True, 7, [40, 13], [33, 13], 1),           # pairs that share no lane layout
    (BF, (16, 8), 2, False, True, 5, [9, 70], [9, 70], 0),
    (BF, (2, 1), 0, False, True, 33, [65], [65], 0),
    (F32, (16, 8), 128, False, True, 16, [333, 1, 0, 12], [333, 1, 0, 12], 0),
    (F32, (16, 8), 32, True, False, 0, [57, 57], [57, 20], 2),
    (F32, (1, 1), 126, False, True, 1, [3, 300], [3, 300], 0),
    (F32, (8, 2), 8, False, True, 48, [100000 // 48, 2], None, 0),
    (BF, (32, 32), 128, True, True, 256, [5000], [5000], 0),
]


@pytest.mark.parametrize("case", range(len(ROTATE)))
def test_rotate(case):
    dtype, (Hq, Hkv), rot, pairs, norm, page, n_ctx, new, lead = ROTATE[case]
    g = torch.Generator().manual_seed(100 + case)
    B = len(n_ctx)
    q_start = None if new is None else _starts(new, lead)
    rows = B if new is None else q_start[-1] + 2                         # and two rows of nobody
    cap = max(n_ctx) + (3 if page else 0)
    kp, vp, table = _cache(g, B, Hkv, max(cap, 1), page, dtype)
    fused = _normal(g, rows, Hq + 2 * Hkv, D, dtype=dtype)
    q, k, v = fused[:, :Hq], fused[:, Hq:Hq + Hkv], fused[:, Hq + Hkv:]
    wq, wk = ((_normal(g, D, dtype=F32) * 0.3 + 1).to(dtype) for _ in range(2)) if norm else (None, None)
    inv = 1e6 ** (-torch.arange(rot // 2, dtype=torch.float64) / max(rot // 2, 1))
    d = kvr.make_desc(B, Hq, Hkv, 1, 1, dtype)
    f_d, kp_d, vp_d, table_d, wq_d, wk_d, inv_d = _dev(fused, kp, vp, table, wq, wk, inv)
    pages = kvr.make_pages(d, kp_d, vp_d, table_d)
    turn = kvr.make_rotation(d, inv_d if rot else None, q_weight=wq_d, k_weight=wk_d, eps=1e-6, pairs=pairs)
    q_out, k_out = torch.full((rows, Hq, D), 7.0, dtype=dtype).cuda(), torch.full((rows, Hkv, D), 7.0, dtype=dtype).cuda()
    qs = None if q_start is None else torch.tensor(q_start, dtype=torch.int32).cuda()
    nc = torch.tensor(n_ctx, dtype=torch.int32).cuda()
    kvr.kvr_rotate(d, turn, f_d[:, :Hq], f_d[:, Hq:Hq + Hkv], f_d[:, Hq + Hkv:], rows, qs, nc, q_out, k_out, pages)
    torch.cuda.synchronize()
    mine = torch.zeros(rows, dtype=torch.bool)
    pos = torch.zeros(rows, dtype=torch.long)
    kp0, vp0 = kp.clone(), vp.clone()
    stored = {}
    for b, (r0, y) in enumerate(R.spans(B, rows, q_start)):
        mine[r0:r0 + y] = True
        pos[r0:r0 + y] = torch.arange(n_ctx[b] - y, n_ctx[b])
        for r in range(r0, r0 + y):
            if 0 <= int(pos[r]) < R.capacity(kp, table):
                stored[R.token_row(kp, table, b, int(pos[r]))] = r
    for x, w, got in ((q, wq, q_out), (k, wk, k_out)):
        ref, size = R.rotate(x, w, pos, inv if rot else None, 1e-6, pairs)
        err = (got.cpu().double() - ref).abs()
        assert bool((err <= R.rotate_bound(ref, size, dtype))[mine].all()), float(err[mine].max())
        assert bool((got.cpu()[~mine] == 7.0).all())
    # the cache: what k_out holds and v as it was, at the rows' places and nowhere else
    ko = k_out.cpu()
    for (page_i, row), r in stored.items():
        kp0[page_i, :, row], vp0[page_i, :, row] = ko[r], v[r]
    assert torch.equal(kp_d.cpu(), kp0) and torch.equal(vp_d.cpu(), vp0)


def test_rotate_in_place_parts_and_pages_that_are_not_there():
    """q alone, k alone, in place; rows past the cache, and pages outside the pools, are stored nowhere."""
    g = torch.Generator().manual_seed(5)
    B, Hq, Hkv, dtype = 4, 8, 2, BF
    d = kvr.make_desc(B, Hq, Hkv, 1, 1, dtype)
    q, k, v = (_normal(g, B, h, D, dtype=dtype).cuda() for h in (Hq, Hkv, Hkv))
    inv = (1e4 ** (-torch.arange(64, dtype=torch.float64) / 64)).cuda()
    turn = kvr.make_rotation(d, inv)
    nc = torch.tensor([5, 33, 0, 20], dtype=torch.int32).cuda()          # 33 > 2 pages of 16; 0: position -1
    q_out, k_out = torch.empty_like(q), torch.empty_like(k)
    kvr.kvr_rotate(d, turn, q, None, None, B, None, nc, q_out)
    kvr.kvr_rotate(d, turn, None, k, None, B, None, nc, None, k_out)
    q2, k2 = q.clone(), k.clone()
    kvr.kvr_rotate(d, turn, q2, k2, v, B, None, nc, q2, k2)
    assert torch.equal(q2, q_out) and torch.equal(k2, k_out)
    ref, size = R.rotate(q.cpu(), None, nc.cpu() - 1, inv.cpu(), 0, False)
    assert bool(((q_out.cpu().double() - ref).abs() <= R.rotate_bound(ref, size, dtype)).all())
    pools = [torch.zeros(6, Hkv, 16, D, dtype=dtype).cuda() for _ in range(2)]
    table = torch.tensor([[3, 1], [0, 2], [4, 4], [5, 6]], dtype=torch.int32).cuda()      # 6: no page
    kvr.kvr_rotate(d, turn, q, k, v, B, None, nc, q_out, None, kvr.make_pages(d, *pools, table))
    want = [torch.zeros_like(p) for p in pools]
    want[0][3, :, 4], want[1][3, :, 4] = k_out[0], v[0]
    assert torch.equal(pools[0], want[0]) and torch.equal(pools[1], want[1])


# ---------------------------------------------------------------------------
def _attend(which, d, q, rows, qs, nc, pages, window, n_sink, scores, n_cap, ws_fill=255):
    out = torch.full_like(q, 7.0)
    if which == "paged":
        n = kvr.kvr_attend_paged_workspace_size(d, pages, window, n_sink, scores is not None)
    else:
        n = kvr.kvr_attend_prompt_workspace_size(d, rows, pages, window, n_sink, scores is not None)
    ws = torch.full((max(n, 256),), ws_fill, dtype=torch.uint8, device="cuda")
    if which == "paged":
        kvr.kvr_attend_paged(d, q, nc, pages, window, n_sink, out, scores, n_cap, ws)
    else:
        kvr.kvr_attend_prompt(d, q, rows, qs, nc, pages, window, n_sink, out, scores, n_cap, ws)
    return out


def _check(which, dtype, heads, page, n_ctx, new, window, n_sink, n_cap, *, lead=0, seed=0, scale=None, wild=None, edit=None):
    """One call against float64; wild: a value for every token that no query sees; edit(kp, vp, table): changes first."""
    Hq, Hkv = heads
    g = torch.Generator().manual_seed(1000 + seed)
    B = len(n_ctx)
    q_start = None if new is None else _starts(new, lead)
    rows = B if new is None else q_start[-1] + 2
    kp, vp, table = _cache(g, B, Hkv, max(max(n_ctx), 1) + (2 if page else 0), page, dtype)
    q = _normal(g, rows, Hq, D, dtype=dtype)
    kp[..., :4] *= 3
    if edit is not None:
        edit(kp, vp, table)
    if wild is not None:
        keep = torch.zeros(kp.shape[0], kp.shape[2], dtype=torch.bool)
        for b, (_, y) in enumerate(R.spans(B, rows, q_start)):
            n = min(n_ctx[b], R.capacity(kp, table))
            lo = n - y
            for j in range(n):
                if window == 0 or j > lo - window or j < n_sink:
                    pr = R.token_row(kp, table, b, j)
                    if pr is not None:
                        keep[pr] = True
        kp.transpose(1, 2)[~keep] = wild
        vp.transpose(1, 2)[~keep] = wild
    d = kvr.make_desc(B, Hq, Hkv, 1, 1, dtype, softmax_scale=scale)
    old = torch.rand(B, Hkv, n_cap, generator=g)
    q_d, kp_d, vp_d, table_d, sc = _dev(q, kp, vp, table, old)
    pages = kvr.make_pages(d, kp_d, vp_d, table_d)
    qs = None if q_start is None else torch.tensor(q_start, dtype=torch.int32).cuda()
    nc = torch.tensor(n_ctx, dtype=torch.int32).cuda()
    out = _attend(which, d, q_d, rows, qs, nc, pages, window, n_sink, sc, n_cap)
    alone = _attend(which, d, q_d, rows, qs, nc, pages, window, n_sink, None, 0, ws_fill=0)
    torch.cuda.synchronize()
    ref = R.attend(q, kp, vp, table, n_ctx, q_start, d.softmax_scale, window, n_sink, n_cap, Hkv)
    tol, tol_s = R.attend_bounds(ref, dtype, old)
    got = out.cpu().double()
    fin = torch.isfinite(ref["out"])
    assert torch.equal(torch.isfinite(got)[ref["rows"]], fin[ref["rows"]])
    err = torch.where(fin, (got - ref["out"]).abs(), torch.zeros_like(got))
    bad = (err > tol) & fin & ref["rows"][:, None, None]
    assert not bool(bad.any()), (int(bad.sum()), float(err[ref["rows"]].max()), bad.nonzero()[:4].tolist())
    assert bool((got[~ref["rows"]] == 7.0).all())
    err = (sc.cpu().double() - old.double() - ref["scores"]).abs()
    assert bool((err <= tol_s).all()), (float(err.max()), (err > tol_s).nonzero()[:4].tolist())
    assert torch.equal(sc.cpu()[ref["scores"] == 0], old[ref["scores"] == 0])
    err = torch.where(fin, (alone.cpu().double() - ref["out"]).abs(), torch.zeros_like(got))
    assert not bool(((err > tol) & fin & ref["rows"][:, None, None]).any())
    return out, sc


HEADS = [(32, 8), (8, 8), (16, 8), (64, 8), (2, 1), (4, 4)]


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("heads", [(8, 8), (4, 2), (8, 2), (16, 2)])
@pytest.mark.parametrize("n", [1, 15, 64, 257, 1000])
def test_one_token(dtype, heads, n):
    _check("paged", dtype, heads, 16, [n, max(1, n // 3)], None, 0, 0, n + 1, seed=n)


ONE = [  # dtype, heads, page, lengths, window, sinks, n_cap
    (BF, (32, 8), 0, [1000], 0, 0, 1000),
    (BF, (8, 2), 24, [0, 1, 2, 16, 17, 0], 0, 0, 30),
    (BF, (8, 2), 1, [77, 5], 0, 0, 40),
    (BF, (16, 2), 100, [2000, 1, 700], 64, 4, 2100),
    (BF, (8, 1), 64, [5000, 4999], 1000, 1, 5000),
    (BF, (4, 4), 7, [300, 299, 20], 1, 0, 300),
    (BF, (4, 2), 16, [900], 17, 1000, 900),
    (BF, (8, 8), 256, [3000], 500, 33, 100),
    (F32, (8, 2), 0, [400, 3], 0, 0, 400),
    (F32, (16, 2), 24, [0, 1200, 33], 100, 16, 1300),
    (F32, (8, 8), 16, [1025], 0, 0, 1025),
    (F32, (2, 1), 5, [64, 65, 66], 16, 1, 70),
    (BF, (32, 8), 64, [20000], 0, 0, 20000),
    (F32, (4, 1), 64, [17000], 0, 0, 17000),
]


@pytest.mark.parametrize("case", range(len(ONE)))
def test_one_token_cases(case):
    dtype, heads, page, n, window, sink, n_cap = ONE[case]
    _check("paged", dtype, heads, page, n, None, window, sink, n_cap, seed=50 + case)
    if max(n) <= 2100:
        _check("paged", dtype, heads, page, n, None, window, sink, n_cap, seed=80 + case, wild=float("nan"))


PROMPT = [  # dtype, heads, page, lengths, new, window, sinks, n_cap, rows of nobody before
    (BF, (8, 2), 0, [1], [1], 0, 0, 1, 0),
    (BF, (8, 2), 0, [130, 64], [130, 64], 0, 0, 130, 0),
    (BF, (8, 2), 16, [200, 0, 1, 77], [200, 0, 1, 70], 0, 0, 210, 3),
    (BF, (8, 8), 24, [513, 65], [513, 64], 0, 0, 500, 0),
    (BF, (4, 2), 100, [300, 299], [300, 17], 32, 4, 300, 0),
    (BF, (16, 2), 64, [400], [400], 100, 1, 400, 0),
    (BF, (16, 2), 7, [90, 33], [2, 33], 1, 0, 90, 0),
    (BF, (8, 1), 32, [1500, 1400], [3, 40], 0, 0, 1500, 0),
    (BF, (8, 2), 64, [700], [600], 64, 70, 700, 0),
    (BF, (4, 4), 1, [50, 3], [50, 3], 7, 2, 50, 0),
    (BF, (8, 2), 16, [40, 10], [60, 12], 0, 0, 50, 0),          # more new rows than tokens: positions below 0
    (F32, (8, 2), 0, [130, 64], [130, 64], 0, 0, 130, 0),
    (F32, (8, 8), 24, [200, 0, 1, 77], [200, 0, 1, 70], 0, 0, 150, 2),
    (F32, (16, 2), 16, [300], [300], 20, 4, 300, 0),
    (F32, (4, 4), 50, [600, 3], [9, 3], 0, 0, 600, 0),
]


@pytest.mark.parametrize("wild", [None, float("nan"), float("-inf")])
@pytest.mark.parametrize("case", range(len(PROMPT)))
def test_prompt(case, wild):
    dtype, heads, page, n, new, window, sink, n_cap, lead = PROMPT[case]
    _check("prompt", dtype, heads, page, n, new, window, sink, n_cap, lead=lead, seed=case, wild=wild)


LONG = [  # many tiles that all columns see whole, and few columns over many tokens, whose tiles are split
    (BF, (8, 2), 0, [1100], [1100], 0, 0, 1100),
    (BF, (8, 2), 16, [1100, 300], [1100, 290], 0, 0, 1100),
    (BF, (4, 4), 64, [900], [900], 300, 5, 900),
    (BF, (8, 1), 5, [700, 20], [700, 20], 0, 0, 700),
    (BF, (8, 2), 16, [6000, 5001], [3, 20], 0, 0, 6000),
    (BF, (8, 8), 64, [9000], [1], 0, 0, 9000),
    (BF, (8, 2), 7, [4100], [33], 0, 0, 4100),
    (BF, (4, 2), 128, [5000, 4000, 0], [130, 2, 0], 3000, 70, 5000),
    (F32, (4, 2), 16, [1500, 600], [20, 600], 0, 0, 1500),
]


@pytest.mark.parametrize("case", range(len(LONG)))
def test_long_prompts(case):
    dtype, heads, page, n, new, window, sink, n_cap = LONG[case]
    _check("prompt", dtype, heads, page, n, new, window, sink, n_cap, seed=200 + case)


PARTS = [  # heads, page, lengths, new, window, sinks: few columns, whose tokens several workgroups share
    ((8, 2), 16, [1000] * 8, [16] * 8, 0, 0),
    ((8, 2), 16, [1200, 0, 3, 2500], [16, 0, 3, 1], 0, 0),
    ((6, 3), 24, [1500, 130], [40, 2], 0, 0),                   # three kv heads: no whole number of them in the launch
    ((8, 1), 16, [300] * 69 + [2000], [0] * 69 + [4], 0, 0),    # one sequence of many has new tokens
    ((8, 2), 16, [129, 128], [1, 128], 0, 0),
    ((16, 2), 64, [3000], [70], 700, 130),
    ((4, 4), 0, [2000], [200], 0, 0),
]


@pytest.mark.parametrize("case", range(len(PARTS)))
def test_parts_of_few_columns(case):
    heads, page, n, new, window, sink = PARTS[case]
    _check("prompt", BF, heads, page, n, new, window, sink, max(n), seed=300 + case, lead=2)


@pytest.mark.parametrize("which", ["prompt", "paged"])
@pytest.mark.parametrize("dtype", [BF, F32])
def test_many_sequences(which, dtype):
    """More sequences than a wave has lanes, empty ones and ones without new tokens among them."""
    n = [(37 * b) % 90 for b in range(150)]
    new = [min(x, (11 * b) % 7) for b, x in enumerate(n)] if which == "prompt" else None
    _check(which, dtype, (4, 2), 16, n, new, 0, 0, 90, seed=77)
    _check(which, dtype, (4, 2), 16, n, new, 20, 2, 90, seed=78, lead=4 if new else 0)


@pytest.mark.parametrize("dtype,heads,n", [(BF, (8, 2), 1000), (BF, (16, 2), 500), (BF, (2, 2), 700), (F32, (8, 2), 800), (F32, (16, 2), 300)])
def test_many_short_caches(dtype, heads, n):
    """A unit to a workgroup with several tiles a wave; the longest of them as much as the cache holds."""
    lens = [max(0, n - 29 * b) for b in range(36)]
    _check("paged", dtype, heads, 16, lens, None, 0, 0, n, seed=91)
    _check("paged", dtype, heads, 24, lens, None, 100, 20, n - 5, seed=92, wild=float("nan"))


@pytest.mark.parametrize("page", [8, 16, 7, 64])
def test_a_page_in_the_middle_is_not_there(page):
    """Where the tokens are many, and few columns see them all, whole and split."""
    def edit(kp, vp, table):
        table[0, (400 // page) + 1] = -1
        table[0, 900 // page] = kp.shape[0] + 5
    for n, new in ((1000, 8), (1000, 400), (2600, 4)):
        _check("prompt", BF, (8, 2), page, [n], [new], 0, 0, n, seed=31 + page, edit=edit)
    _check("paged", BF, (8, 2), page, [1000], None, 0, 0, 1000, seed=31 + page, edit=edit)


@pytest.mark.parametrize("which", ["prompt", "paged"])
@pytest.mark.parametrize("dtype", [BF, F32])
def test_pages_that_are_not_there(which, dtype):
    """Pages outside the pools hold no tokens: in front (a window gave them back), in the middle, and all of them."""
    def edit(kp, vp, table):
        table[0, :3] = -1
        table[1, 2] = kp.shape[0]
        table[2, :] = -7
        table[3, :] = table[0, :]                       # two sequences share their pages
    new = [100, 90, 50, 20] if which == "prompt" else None
    _check(which, dtype, (8, 2), 16, [100, 90, 50, 95], new, 0, 0, 100, seed=7, edit=edit)
    _check(which, dtype, (8, 2), 16, [100, 90, 50, 95], new, 33, 5, 100, seed=8, edit=edit)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("value", [float("inf"), float("nan")])
def test_values_that_later_queries_alone_see(dtype, value):
    """A value that is not finite reaches the queries that see it and no other: later ones, with a window neither those
    that have left it behind."""
    def edit(kp, vp, table):
        for j in (5, 40, 64, 100):
            vp[int(table[0, j // 16]), 1, j % 16, 3:60] = value
    _check("prompt", dtype, (8, 2), 16, [130], [130], 0, 0, 130, seed=3, edit=edit)
    _check("prompt", dtype, (8, 2), 16, [130], [130], 20, 2, 130, seed=4, edit=edit)


# the calls' routes: few tokens, many, and few columns over many
ROUTES = [("prompt", BF, [100, 32], [100, 32]), ("prompt", BF, [3000, 32], [4, 3]), ("prompt", F32, [130, 32], [130, 32]),
          ("paged", BF, [100, 32], None), ("paged", BF, [3000, 32], None), ("paged", F32, [100, 32], None), ("paged", F32, [3000, 32], None)]


def _odd_call(which, dtype, n, new, change):
    """-> result of a call on operands that change(q, kp, vp, table) has altered, and of float64 on what it returns."""
    g = torch.Generator().manual_seed(17)
    q_start = None if new is None else _starts(new)
    rows = 2 if new is None else q_start[-1]
    kp, vp, table = _cache(g, 2, 2, max(n), 16, dtype)
    q = _normal(g, rows, 8, D, dtype=dtype)
    d = kvr.make_desc(2, 8, 2, 1, 1, dtype)
    as_if = change(q, kp, vp, table)
    old = torch.rand(2, 2, max(n), generator=g)
    q_d, kp_d, vp_d, table_d, sc = _dev(q, kp, vp, table, old)
    qs = None if q_start is None else torch.tensor(q_start, dtype=torch.int32).cuda()
    nc = torch.tensor(n, dtype=torch.int32).cuda()
    out = _attend(which, d, q_d, rows, qs, nc, kvr.make_pages(d, kp_d, vp_d, table_d), 0, 0, sc, max(n))
    ref = R.attend(*as_if, n, q_start, d.softmax_scale, 0, 0, max(n), 2)
    tol, tol_s = R.attend_bounds(ref, dtype, old)
    off = (out.cpu().double() - ref["out"]).abs() / tol
    off_s = (sc.cpu().double() - old.double() - ref["scores"]).abs() / tol_s
    return out.cpu(), sc.cpu(), off, off_s, q_start


@pytest.mark.parametrize("case", range(len(ROUTES)))
def test_logits_of_minus_infinity(case):
    """Tokens whose logit is -inf for every head weigh nothing, also where they come first or fill tiles; a query that sees
    no others yields zeros (the second sequence)."""
    which, dtype, n, new = ROUTES[case]

    def change(q, kp, vp, table):
        q[..., 0] = -1
        less = table.clone()
        for b, pages in ((0, [0, 1, 2, 3, 5]), (1, [0, 1])):
            for i in pages:
                kp[int(table[b, i]), :, :, 0] = float("inf")
                less[b, i] = -1
        return q, kp, vp, less

    out, sc, off, off_s, q_start = _odd_call(which, dtype, n, new, change)
    assert float(off.max()) <= 1 and float(off_s.max()) <= 1
    second = out[1:] if new is None else out[q_start[1]:]
    assert not bool(second.any())


@pytest.mark.parametrize("case", range(len(ROUTES)))
def test_nan_in_a_query_or_a_key_stays_with_who_sees_it(case):
    which, dtype, n, new = ROUTES[case]
    first = n[0] - (1 if new is None else new[0])                # position of the first sequence's first row
    row, head = (0, 3) if new is None else (new[0] // 2, 3)

    def query(q, kp, vp, table):
        clean = q.clone(), kp, vp, table
        q[row, head, 77] = float("nan")
        return clean

    out, sc, off, off_s, _ = _odd_call(which, dtype, n, new, query)
    assert bool(out[row, head].isnan().all())
    off[row, head] = 0
    assert float(off.max()) <= 1
    sees = first + row + 1
    assert bool(sc[0, 0, :sees].isnan().all())
    off_s[0, 0, :sees] = 0
    assert float(off_s.max()) <= 1

    j = max(first + row, 0)                                      # a token that the rows from `row` on see

    def key(q, kp, vp, table):
        clean = q, kp.clone(), vp, table
        kp[int(table[0, j // 16]), 1, j % 16, 5] = float("nan")
        return clean

    out, sc, off, off_s, q_start = _odd_call(which, dtype, n, new, key)
    end = 1 if new is None else q_start[1]
    assert bool(out[row:end, 4:].isnan().all())
    off[row:end, 4:] = 0
    assert float(off.max()) <= 1
    assert bool(sc[0, 1, :n[0]].isnan().all())
    off_s[0, 1] = 0
    assert float(off_s.max()) <= 1


@pytest.mark.parametrize("which", ["prompt", "paged"])
@pytest.mark.parametrize("scale", [0.0, -0.05, 0.5])
def test_scales(which, scale):
    """Any factor, also one that turns the order of the logits round or makes them all alike."""
    _check(which, BF, (8, 2), 16, [150, 40], [150, 30] if which == "prompt" else None, 0, 0, 150, seed=9, scale=scale)
    _check(which, BF, (8, 2), 16, [150, 40], [150, 30] if which == "prompt" else None, 16, 3, 150, seed=9, scale=scale)


@pytest.mark.parametrize("which", ["prompt", "paged"])
def test_lengths_past_the_cache_are_clamped(which):
    g = torch.Generator().manual_seed(2)
    d = kvr.make_desc(2, 8, 2, 1, 1, BF)
    kp, vp, table = _cache(g, 2, 2, 64, 16, BF)
    q = _normal(g, 2, 8, D, dtype=BF)
    q, kp, vp, table = _dev(q, kp, vp, table)
    pages = kvr.make_pages(d, kp, vp, table)
    res = []
    for n in ([64, 64], [2 ** 31 - 1, 65]):
        nc = torch.tensor(n, dtype=torch.int32).cuda()
        sc = torch.zeros(2, 2, 70).cuda()
        res.append((_attend(which, d, q, 2, None, nc, pages, 0, 0, sc, 70), sc))
    assert torch.equal(res[0][0], res[1][0]) and torch.equal(res[0][1], res[1][1])
    nc = torch.tensor([-5, -2 ** 31 + 1], dtype=torch.int32).cuda()
    sc = torch.zeros(2, 2, 70).cuda()
    assert bool((_attend(which, d, q, 2, None, nc, pages, 0, 0, sc, 70) == 0).all()) and bool((sc == 0).all())


@pytest.mark.parametrize("which", ["prompt", "paged"])
def test_same_result_every_time_and_in_a_graph(which):
    """No order of a sum depends on chance: calls, and replays of a captured call with other work between, agree bit for
    bit, on a stream other than the one that made the tensors too."""
    g = torch.Generator().manual_seed(11)
    n = [3000, 17, 0]
    new = [70, 17, 0] if which == "prompt" else None
    q_start = None if new is None else _starts(new)
    rows = 3 if new is None else q_start[-1]
    d = kvr.make_desc(3, 8, 2, 1, 1, BF)
    kp, vp, table = _cache(g, 3, 2, 3000, 16, BF)
    q, kp, vp, table = _dev(_normal(g, rows, 8, D, dtype=BF), kp, vp, table)
    pages = kvr.make_pages(d, kp, vp, table)
    nc = torch.tensor(n, dtype=torch.int32).cuda()
    qs = None if q_start is None else torch.tensor(q_start, dtype=torch.int32).cuda()
    sc = torch.zeros(3, 2, 3000).cuda()
    first = _attend(which, d, q, rows, qs, nc, pages, 1000, 4, sc, 3000)
    again_sc = torch.zeros_like(sc)
    assert torch.equal(first, _attend(which, d, q, rows, qs, nc, pages, 1000, 4, again_sc, 3000))
    assert torch.equal(sc, again_sc)
    if which == "paged":
        size = kvr.kvr_attend_paged_workspace_size(d, pages, 1000, 4, True)
    else:
        size = kvr.kvr_attend_prompt_workspace_size(d, rows, pages, 1000, 4, True)
    ws = torch.zeros(max(size, 256), dtype=torch.uint8, device="cuda")
    out, acc = torch.zeros_like(q), torch.zeros_like(sc)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        if which == "paged":
            kvr.kvr_attend_paged(d, q, nc, pages, 1000, 4, out, acc, 3000, ws)
        else:
            kvr.kvr_attend_prompt(d, q, rows, qs, nc, pages, 1000, 4, out, acc, 3000, ws)
    for _ in range(4):
        out.fill_(3.0)
        acc.zero_()
        ws.random_(0, 255)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, first) and torch.equal(acc, sc)
        _ = (out.float() @ out.float().transpose(1, 2)).sum().item()


def test_prompt_of_one_token_is_the_paged_call():
    """Both calls give the same function: within the bounds of their roundings."""
    g = torch.Generator().manual_seed(21)
    d = kvr.make_desc(2, 8, 2, 1, 1, BF)
    kp, vp, table = _cache(g, 2, 2, 500, 16, BF)
    q, kp, vp, table = _dev(_normal(g, 2, 8, D, dtype=BF), kp, vp, table)
    pages = kvr.make_pages(d, kp, vp, table)
    nc = torch.tensor([500, 31], dtype=torch.int32).cuda()
    a = _attend("prompt", d, q, 2, None, nc, pages, 0, 0, None, 0).float()
    b = _attend("paged", d, q, 2, None, nc, pages, 0, 0, None, 0).float()
    ref = R.attend(q.cpu(), kp.cpu(), vp.cpu(), table.cpu(), [500, 31], None, d.softmax_scale, 0, 0, 1, 2)
    tol, _ = R.attend_bounds(ref, BF)
    assert bool(((a - b).abs().cpu().double() <= 2 * tol).all())


def test_offsets_past_32_bits():
    """Pools of more than 2^31 elements: tokens on the last pages."""
    pages_n, Hkv, ps = 2200, 8, 1024                       # 2200 x 8 x 1024 x 128 = 2.3e9 elements, 4.6 GB a pool
    d = kvr.make_desc(1, 8, 8, 1, 1, BF)
    kp = torch.zeros(pages_n, Hkv, ps, D, dtype=BF, device="cuda")
    vp = torch.zeros_like(kp)
    g = torch.Generator().manual_seed(1)
    k, v = _normal(g, Hkv, ps, D, dtype=BF), _normal(g, Hkv, ps, D, dtype=BF)
    kp[pages_n - 1], vp[pages_n - 1] = k.cuda(), v.cuda()
    table = torch.tensor([[pages_n - 1]], dtype=torch.int32).cuda()
    pages = kvr.make_pages(d, kp, vp, table)
    n = 1000
    q = _normal(g, 5, 8, D, dtype=BF)
    nc = torch.tensor([n], dtype=torch.int32).cuda()
    qs = torch.tensor([0, 5], dtype=torch.int32).cuda()
    out = _attend("prompt", d, q.cuda(), 5, qs, nc, pages, 0, 0, None, 0)
    ref = R.attend(q, k[None], v[None], None, [n], [0, 5], d.softmax_scale, 0, 0, 1, 8)
    tol, _ = R.attend_bounds(ref, BF)
    assert bool(((out.cpu().double() - ref["out"]).abs() <= tol).all())
    one = _attend("paged", d, q[4:].contiguous().cuda(), 1, None, nc, pages, 0, 0, None, 0)
    assert bool(((one.cpu().double() - ref["out"][4:]).abs() <= tol[4:]).all())
    turn = kvr.make_rotation(d)
    x = _normal(g, 1, 24, D, dtype=BF).cuda()
    kvr.kvr_rotate(d, turn, x[:, :8], x[:, 8:16], x[:, 16:], 1, None, nc, torch.empty_like(x[:, :8]), None, pages)
    assert torch.equal(kp[pages_n - 1, :, n - 1], x[0, 8:16]) and torch.equal(vp[pages_n - 1, :, n - 1], x[0, 16:])

"""Windows over groups in the kernels that share (tests/test_shared_routes_cpu.py sees that these sizes take them): several new rows a
sequence with 1, 2, 4 and 8 heads a key head, pages of odd sizes, ends that the join attends to, and a captured call."""
import math

import pytest
import torch

from paper_2512_17917_amd import binding as kvr
from tests import cache_ref as R
from tests.test_gpu_cache_state import _near
from tests.test_gpu_shared import BF, D, F32, Batch, _many

pytestmark = [pytest.mark.gpu, pytest.mark.timeout(300)]

WINDOWS = [  # rows of a sequence at most, groups, heads, page, window, first tokens
    (3, [_many(3, 40, 900), _many(3, 20, 640)], (16, 8), 7, 600, 20),
    (5, [_many(5, 50, 1700), _many(5, 40, 1500)], (8, 2), 7, 1500, 0),
    (3, [_many(3, 60, 1400), _many(3, 45, 1500)], (16, 2), 24, 1300, 130),
    (2, [_many(2, 40, 1300)], (64, 8), 5, 1100, 4),
    (4, [_many(4, 70, 900)], (8, 8), 16, 700, 64),
    (1, [_many(1, 100, 500), _many(1, 60, 64)], (32, 8), 16, 300, 9),
    (1, [_many(1, 150, 300), _many(1, 50, 70)], (16, 8), 7, 30, 230),
]


def batch(case, dtype):
    most, groups, heads, page, window, sink = WINDOWS[case]
    return Batch(groups, heads, page, dtype, 160 + case, rows=most > 1, room=0), window, sink


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("case", range(len(WINDOWS)))
def test_windows(case, dtype):
    """Also with pages that are not there, and values that are not finite where some columns see them and others do not."""
    b, window, sink = batch(case, dtype)
    b.check(window, sink)
    page = b.page
    for i, (c, (first, end)) in enumerate(zip(b.common, zip(b.start, b.start[1:]))):
        at = max(c - window, 0) // page + 1                      # a page of what is shared
        if i % 2 == 0 and (at + 1) * page <= c:
            b.table[first:end, at] = -1
        for j, what in ((c - 1, math.nan), (max(c - window + 100, 0), math.inf), (sink // 2, -math.inf)):
            for s in range(first, end):                          # (copies of a page that is filled in part have it too)
                at = R.token_row(b.k, b.table, s, j) if j < b.n[s] else None
                if at is not None:
                    b.v[at[0], 1, at[1], 64 + i] = what
        for s, what in ((end - 1, math.inf), (end - 2, math.nan)):
            at = R.token_row(b.k, b.table, s, b.n[s] - 1)
            if at is not None and b.n[s] > c:
                b.v[at[0], 0, at[1], 3] = what
    b.check(window, sink, scores=False)
    b.check(window, sink)


# ---------------------------------------------------------------------------
B_, HQ, HKV, PAGE, WINDOW, SINK, ROWS, TOKENS = 60, 16, 8, 16, 600, 20, 150, 2000
STEPS = [  # groups' starts (three at most), tokens in common, tokens behind them, new rows where there are starts
    ([0, 40, 60, 60], [900, 640, 0], lambda b: 1 + 3 * b, lambda b: 1 + b % 4),
    ([0, 10, 30, 60], [900, 640, 1280], lambda b: 1 + b, lambda b: b % 3),
    ([5, 5, 30, 60], [900, 640, 64], lambda b: 2 * b, lambda b: 1 + b % 2),
    ([0, 0, 0, 0], [0, 0, 0], lambda b: 28 * b, lambda b: 2),
    ([0, 40, 60, 60], [900, 640, 0], lambda b: 1 + 3 * b, lambda b: 1 + b % 4),
]


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("rows", [True, False])
def test_a_captured_call_under_a_window(rows, dtype):
    """Replayed over other lengths, groups and rows; every replay against the eager call, one of them against float64."""
    g = torch.Generator().manual_seed(170)
    d = kvr.make_desc(B_, HQ, HKV, 1, 1, dtype)
    pool = 700
    k, v = (torch.randn(pool, HKV, PAGE, D, generator=g).to(dtype) for _ in range(2))
    table = torch.randint(0, pool, (B_, TOKENS // PAGE), generator=g, dtype=torch.int32)
    table[:, :80] = table[0, :80]                                # all begin with the same 1280 tokens
    kc, vc = k.cuda(), v.cuda()
    pages = kvr.make_pages(d, kc, vc, table.cuda())
    n_rows = ROWS if rows else B_
    q = torch.randn(n_rows, HQ, D, generator=g).to(dtype).cuda()
    i32 = lambda n: torch.zeros(n, dtype=torch.int32, device="cuda")
    n_ctx, q_start, start, common = i32(B_), i32(B_ + 1), i32(4), i32(3)
    groups = kvr.make_groups(start, common)
    out, scores = torch.empty_like(q), torch.empty(B_, HKV, TOKENS, device="cuda")
    ws = torch.empty(kvr.kvr_attend_shared_workspace_size(d, n_rows, pages, groups, WINDOW, SINK, True), dtype=torch.uint8, device="cuda")
    run = lambda: kvr.kvr_attend_shared(d, q, n_rows, q_start if rows else None, n_ctx, pages, groups, WINDOW, SINK, out, scores, TOKENS, ws)
    lens = []

    def set_to(at):
        s, c, more, new = at
        of = [next((c[i] for i in range(3) if s[i] <= b < s[i + 1]), 300) for b in range(B_)]
        n, starts = [x + more(b) + 3 for b, x in enumerate(of)], [0]
        for b in range(B_):
            starts.append(starts[-1] + new(b))
        assert starts[-1] <= ROWS and max(n) <= TOKENS
        for to, x in ((n_ctx, n), (q_start, starts), (start, s), (common, c)):
            to.copy_(torch.tensor(x, dtype=torch.int32))
        out.fill_(3.0)
        scores.fill_(0.5)
        lens[:] = [n, starts if rows else None]
    set_to(STEPS[0])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run()
    want = []
    for s in STEPS:
        set_to(s)
        ws.fill_(255)
        run()
        want.append((out.clone(), scores.clone(), *lens))
    assert torch.equal(want[0][0], want[-1][0]) and torch.equal(want[0][1], want[-1][1])
    for s, (o, sc, *_) in zip(STEPS, want):
        set_to(s)
        ws.random_(0, 255)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, o) and torch.equal(scores, sc)
        _ = (out.float() @ out.float().transpose(1, 2)).sum().item()
    o, sc, n, starts = want[1]
    ref = R.attend(q.cpu(), k, v, table, n, starts, d.softmax_scale, WINDOW, SINK, TOKENS, HKV)
    tol = _near(o, ref, dtype, torch.full((B_, HKV, TOKENS), 0.5))
    assert bool(((sc.cpu().double() - 0.5 - ref["scores"]).abs() <= tol).all())

"""What kvr.h says of kvr_attend_prompt and kvr_attend_paged alike: NaN among the logits that a query sees reaches the scores of
all tokens that it sees, also of those whose own logit is -Inf, and of no others; the calls without scores keep the same rules."""
import pytest
import torch

from paper_2512_17917_amd import binding as kvr
from tests import cache_ref as R
from tests.test_gpu_cache_ops import _attend, _cache, _dev, _normal, _starts

pytestmark = [pytest.mark.gpu, pytest.mark.timeout(300)]
D = 128
BF, F32 = torch.bfloat16, torch.float32

# few tokens, many; a workgroup a unit with several tiles a wave (many sequences); few columns over many tokens
ROUTES = [("prompt", BF, 1, [100], [100]), ("prompt", BF, 1, [3000], [4]), ("prompt", F32, 1, [130], [130]), ("paged", BF, 1, [100], None),
          ("paged", BF, 1, [3000], None), ("paged", F32, 1, [100], None), ("paged", F32, 1, [3000], None), ("paged", BF, 40, [900] * 40, None),
          ("paged", F32, 40, [500] * 40, None)]


@pytest.mark.parametrize("window,sink", [(0, 0), (60, 5)])
@pytest.mark.parametrize("case", range(len(ROUTES)))
def test_nan_reaches_the_scores_of_seen_tokens_of_logit_minus_infinity(case, window, sink):
    """The first sequence's second kv head: a NaN key near its end, whole pages of keys whose logits are -Inf, one page that is
    not there."""
    which, dtype, B, n, new = ROUTES[case]
    g = torch.Generator().manual_seed(40 + case)
    q_start = None if new is None else _starts(new)
    rows = B if new is None else q_start[-1]
    kp, vp, table = _cache(g, B, 2, max(n) + 30, 16, dtype)
    q = _normal(g, rows, 8, D, dtype=dtype)
    q[..., 0] = -1
    last = n[0] - 1
    low = [0, (last - 30) // 16, last // 16]                     # pages of -Inf: the first tokens, behind the window's start, the end
    gone = (last - 50) // 16 if window == 0 else (last - 20) // 16
    low = [i for i in low if i != gone]
    for i in low:
        kp[int(table[0, i]), 1, :, 0] = float("inf")
    table[0, gone] = -1
    at = next(j for j in range(last, 0, -1) if j // 16 not in low and j // 16 != gone)
    kp[int(table[0, at // 16]), 1, at % 16, 5] = float("nan")
    d = kvr.make_desc(B, 8, 2, 1, 1, dtype)
    n_cap = max(n) + 20
    old = torch.rand(B, 2, n_cap, generator=g)
    q_d, kp_d, vp_d, table_d, sc = _dev(q, kp, vp, table, old)
    qs = None if q_start is None else torch.tensor(q_start, dtype=torch.int32).cuda()
    nc = torch.tensor(n, dtype=torch.int32).cuda()
    pages = kvr.make_pages(d, kp_d, vp_d, table_d)
    out = _attend(which, d, q_d, rows, qs, nc, pages, window, sink, sc, n_cap).cpu()
    y = 1 if new is None else new[0]
    seen = torch.zeros(n_cap, dtype=torch.bool)                  # by a query that sees the NaN
    for p in range(max(at, n[0] - y), n[0]):
        if window and at <= p - window and at >= sink:
            continue
        for j in range(p + 1):
            if (window == 0 or j > p - window or j < sink) and j // 16 != gone:
                seen[j] = True
    assert bool(seen.any()) and any(bool(seen[16 * i:16 * i + 16].any()) for i in low)
    got = sc[0, 1].cpu()
    assert torch.equal(got.isnan(), seen), (got.isnan() != seen).nonzero()[:8, 0].tolist()
    end = 1 if new is None else q_start[1]
    assert bool(out[end - 1, 4:].isnan().all()) and not bool(out[:, :4].isnan().any())
    assert not bool(sc[0, 0].isnan().any()) and not bool(sc[1:].isnan().any())
    assert torch.equal(got[n[0]:], old[0, 1, n[0]:]) and torch.equal(got[16 * gone:16 * gone + 16], old[0, 1, 16 * gone:16 * gone + 16])


ALONE = [  # which, dtype, heads, page, lengths, new, window, sinks, rows of nobody before
    ("prompt", BF, (8, 2), 16, [200, 0, 1, 77], [200, 0, 1, 70], 0, 0, 3),
    ("prompt", BF, (16, 2), 64, [400], [400], 100, 1, 0),
    ("prompt", BF, (8, 2), 64, [700], [600], 64, 70, 2),
    ("prompt", BF, (8, 2), 16, [6000, 5001], [3, 20], 0, 0, 1),
    ("prompt", BF, (4, 2), 16, [1100], [1100], 300, 5, 0),
    ("prompt", F32, (8, 8), 24, [200, 0, 1, 77], [200, 0, 1, 70], 0, 0, 2),
    ("prompt", F32, (16, 2), 16, [300], [300], 20, 4, 1),
    ("paged", BF, (16, 2), 100, [2000, 1, 700, 0], None, 64, 4, 0),
    ("paged", BF, (8, 2), 16, [130, 5], None, 0, 0, 0),
    ("paged", F32, (8, 2), 24, [0, 1200, 33], None, 100, 16, 0),
]


@pytest.mark.parametrize("wild", [float("nan"), float("-inf")])
@pytest.mark.parametrize("case", range(len(ALONE)))
def test_calls_without_scores_pass_over_what_nobody_sees(case, wild):
    """Every token that no query sees holds NaN or -Inf; one page is not there.  The same bits as with scores, nobody's rows as they
    were."""
    which, dtype, (Hq, Hkv), page, n, new, window, sink, lead = ALONE[case]
    g = torch.Generator().manual_seed(400 + case)
    B = len(n)
    q_start = None if new is None else _starts(new, lead)
    rows = B if new is None else q_start[-1] + 2
    kp, vp, table = _cache(g, B, Hkv, max(n) + 2, page, dtype)
    table[0, (n[0] - 1) // page - 1 if n[0] > 2 * page else 0] = -1
    keep = torch.zeros(kp.shape[0], kp.shape[2], dtype=torch.bool)
    for b, (_, y) in enumerate(R.spans(B, rows, q_start)):
        for j in range(n[b]):
            pr = R.token_row(kp, table, b, j)
            if pr is not None and (window == 0 or j > n[b] - y - window or j < sink):
                keep[pr] = True
    kp.transpose(1, 2)[~keep] = wild
    vp.transpose(1, 2)[~keep] = wild
    q = _normal(g, rows, Hq, D, dtype=dtype)
    d = kvr.make_desc(B, Hq, Hkv, 1, 1, dtype)
    q_d, kp_d, vp_d, table_d = _dev(q, kp, vp, table)
    qs = None if q_start is None else torch.tensor(q_start, dtype=torch.int32).cuda()
    nc = torch.tensor(n, dtype=torch.int32).cuda()
    pages = kvr.make_pages(d, kp_d, vp_d, table_d)
    alone = _attend(which, d, q_d, rows, qs, nc, pages, window, sink, None, 0).cpu()
    sc = torch.zeros(B, Hkv, max(n)).cuda()
    with_scores = _attend(which, d, q_d, rows, qs, nc, pages, window, sink, sc, max(n)).cpu()
    ref = R.attend(q, kp, vp, table, n, q_start, d.softmax_scale, window, sink, 1, Hkv)
    tol, _ = R.attend_bounds(ref, dtype)
    mine = ref["rows"]
    assert bool(torch.isfinite(alone[mine]).all()) and bool((alone[~mine] == 7.0).all())
    assert bool(((alone.double() - ref["out"]).abs() <= tol)[mine].all())
    assert torch.equal(alone, with_scores)

"""Workgroups with more to do than their lists hold: more than 64 pieces of units, more than 128 tiles (24 where pages are not of whole
eights), also where a list ends between a unit's queries and its tokens.  Against float64, sequence by sequence, on the GPU."""
import pytest
import torch

from paper_2512_17917_amd import binding as kvr
from tests import cache_ref as R

pytestmark = [pytest.mark.gpu, pytest.mark.timeout(300)]
D = 128
BF, F32 = torch.bfloat16, torch.float32

CASES = [  # name, dtypes, heads, page, groups, members, tokens in common, own tokens (first, how many more), new rows at most (0: one, without starts)
    ("pieces", (BF, F32), (8, 8), 16, 4200, 1, 0, (257, 40), 0),             # 33600 units of five tiles: 131 and 66 a workgroup, scores' 66
    ("pieces of several rows", (BF,), (64, 8), 8, 3000, 1, 0, (70, 59), 3),  # 24000 of a tile of queries and two of tokens: 94
    ("tiles", (BF,), (32, 32), 8, 1, 2, 131072, (1, 100), 0),                # 65536 tiles: 256 a workgroup
    ("tiles of odd pages", (BF,), (8, 8), 7, 1, 2, 131072, (1, 100), 0),     # 16384: 64
    ("tiles of odd pages, rows", (BF,), (16, 4), 7, 1, 3, 131000, (20, 50), 5),      # 36 columns, one tile of queries
    ("queries", (BF,), (16, 4), 16, 360, 33, 1536, (1, 30), 0),              # 1440 units of two tiles of queries and 24 of tokens: 146
    ("queries of odd pages", (BF,), (16, 4), 7, 360, 33, 200, (1, 30), 0),   # of two and four: 34
]


class Setup:
    """Tables of pages drawn from a small pool; page p's values are in channel p mod 128, and a run of 64 tokens names pages of one
    channel alone, so that a tile that is left out shows."""

    def __init__(self, case):
        _, _, self.heads, self.page, groups, members, common, (own, more), self.most = CASES[case]
        self.groups, self.B = groups, groups * members
        ps = self.page
        self.n = [common + own + (7 * b) % (more + 1) for b in range(self.B)]
        self.y = [1 if not self.most else 1 + b % self.most for b in range(self.B)]
        self.rows = sum(self.y)
        self.start, self.common = [i * members for i in range(groups + 1)], [common] * groups
        self.cols = -(-max(self.n + [200]) // ps)                # (room that makes the call share)
        self.tables = (groups, members, common)

    def table(self, g):
        groups, members, common = self.tables
        i = torch.arange(self.cols) * self.page // 64            # a run of 64 tokens
        lead = torch.randint(0, 3, (groups, 1, self.cols), generator=g) * 128 + (i + 17 * torch.arange(groups)[:, None, None]) % 128
        own = torch.randint(0, 3, (groups, members, self.cols), generator=g) * 128 + (i + 5 * torch.arange(self.B).view(groups, members, 1)) % 128
        whole = torch.arange(self.cols) < common // self.page
        return torch.where(whole, lead, own).view(self.B, self.cols).to(torch.int32)


def _reference(s, q, k, v, table, scale, n_cap):
    Hq, Hkv = s.heads
    G = Hq // Hkv
    out = torch.zeros(s.rows, Hq, D, dtype=torch.float64, device="cuda")
    scores = torch.zeros(s.B, Hkv, n_cap, dtype=torch.float64, device="cuda")
    at = torch.arange(max(s.n), device="cuda")
    page, row = at // s.page, at % s.page
    kd, vd = k.double(), v.double()
    r = 0
    for b, (n, y) in enumerate(zip(s.n, s.y)):
        p = table[b].long()[page[:n]]
        kb, vb = (x[p, :, row[:n]].transpose(0, 1).contiguous() for x in (kd, vd))
        x = q[r:r + y].double().view(y, Hkv, G, D).transpose(0, 1).reshape(Hkv, y * G, D)
        w = torch.matmul(x, kb.transpose(1, 2).contiguous()) * scale
        pos = torch.arange(n - y, n, device="cuda").repeat_interleave(G)[:, None]
        w = torch.softmax(w.masked_fill(at[:n] > pos, float("-inf")), -1)
        out[r:r + y] = torch.matmul(w, vb).view(Hkv, y, G, D).transpose(0, 1).reshape(y, Hq, D)
        scores[b, :, :n] = w.sum(1)[:, :n_cap]
        r += y
    return out, scores


@pytest.mark.parametrize("case,dtype", [(i, dt) for i, c in enumerate(CASES) for dt in c[1]])
def test_lists_that_are_filled_again(case, dtype):
    s = Setup(case)
    g = torch.Generator().manual_seed(180 + case)
    Hq, Hkv = s.heads
    table = s.table(g).cuda()
    pool = 384
    k = torch.randn(pool, Hkv, s.page, D, generator=g).to(dtype).cuda()
    v = torch.zeros(pool, Hkv, s.page, D)
    v[torch.arange(pool), :, :, torch.arange(pool) % 128] = 0.5 + torch.rand(pool, Hkv, s.page, generator=g)
    v = v.to(dtype).cuda()
    q = torch.randn(s.rows, Hq, D, generator=g).to(dtype).cuda()
    # what is shared to the last token: pages that it ends in hold the same there
    groups_, members, common = s.tables
    if common % s.page:
        at, rest = common // s.page, common % s.page
        own = torch.arange(s.B, device="cuda") + pool
        k, v = (torch.cat([x, x[table[:, at].long()]]) for x in (k, v))
        first = own.view(groups_, members)[:, :1].expand(-1, members).reshape(-1)
        for x in (k, v):
            x[own, :, :rest] = x[first, :, :rest]
        table[:, at] = own.to(torch.int32)
    d = kvr.make_desc(s.B, Hq, Hkv, 1, 1, dtype)
    i32 = lambda x: torch.tensor(x, dtype=torch.int32).cuda()
    q_start = None
    if s.most:
        q_start = i32([0] + torch.tensor(s.y).cumsum(0).tolist())
    pages, grp = kvr.make_pages(d, k, v, table), kvr.make_groups(i32(s.start), i32(s.common))
    n_cap = max(s.n) - 1
    out, scores = torch.full((s.rows, Hq, D), 7.0, dtype=dtype).cuda(), torch.zeros(s.B, Hkv, n_cap, device="cuda")
    ws = torch.randint(0, 256, (kvr.kvr_attend_shared_workspace_size(d, s.rows, pages, grp, 0, 0, True),), dtype=torch.uint8, device="cuda")
    kvr.kvr_attend_shared(d, q, s.rows, q_start, i32(s.n), pages, grp, 0, 0, out, scores, n_cap, ws)
    torch.cuda.synchronize()
    ref_out, ref_scores = _reference(s, q, k, v, table, d.softmax_scale, n_cap)
    # (values are not below 0: a sum of sizes is the sum)
    e = 130 * R.U32 * d.softmax_scale * float(q.double().norm(dim=-1).max() * k.double().norm(dim=-1).max())
    tol, tol_s = R.attend_bounds(dict(out=ref_out, weight=ref_out, scores=ref_scores, e=e), dtype)
    err = (out.double() - ref_out).abs()
    assert bool((err <= tol).all()), float((err - tol).max())
    err = (scores.double() - ref_scores).abs()
    assert bool((err <= tol_s).all()), float((err - tol_s).max())

"""kvr_attend_shared against float64 (tests/cache_ref.py), which knows nothing of groups: the sequences' own table rows.

The call goes by the room of a cache: small ones are read by every sequence for itself.  ROOM tokens more than the longest
sequence has (the table's entries for them name no page) make the small batches here take the kernels for long ones."""
import math

import pytest
import torch

from paper_2512_17917_amd import binding as kvr
from tests import cache_ref as R

pytestmark = [pytest.mark.gpu, pytest.mark.timeout(300)]
D = 128
BF, F32 = torch.bfloat16, torch.float32
ROOM = 200000


class Batch:
    """Groups as lists of (tokens, new rows) with the tokens that they have in common: [(common, [(n, y), ...]), ...]; their
    pools, table, lengths and queries on the CPU."""

    def __init__(self, groups, heads, page, dtype, seed, *, lead=0, trail=0, alone=(), rows=True, room=ROOM):
        """alone: sequences of no group, behind the groups; rows: by q_start (else one row a sequence); room: tokens that a
        sequence can hold past its longest."""
        g = self.g = torch.Generator().manual_seed(seed)
        self.dtype, (self.Hq, self.Hkv), self.page = dtype, heads, page
        seqs = [s for _, m in groups for s in m] + list(alone)
        self.n, new = [n for n, _ in seqs], [y for _, y in seqs]
        self.B, self.start, self.common = len(seqs), [0], [c for c, _ in groups]
        for _, m in groups:
            self.start.append(self.start[-1] + len(m))
        self.q_start = None
        self.rows = self.B
        if rows:
            self.q_start = [lead]
            for y in new:
                self.q_start.append(self.q_start[-1] + y)
            self.rows = self.q_start[-1] + trail
        each = -(-(max(self.n) + room) // page) or 1
        table = torch.full((self.B, each), -1, dtype=torch.int32)
        used, copies = 0, []
        of = [i for i, (_, m) in enumerate(groups) for _ in m] + [None] * len(alone)
        whole = {}                                               # a group's pages that are filled by what it has in common
        for b in range(self.B):
            have = -(-self.n[b] // page)
            c = self.common[of[b]] if of[b] is not None else 0
            for i in range(have):
                if of[b] is not None and (i + 1) * page <= c and (of[b], i) in whole:
                    table[b, i] = whole[of[b], i]
                    continue
                table[b, i] = used
                if of[b] is not None and i * page < c:
                    if (of[b], i) in whole:                      # the page that the common tokens end in: a copy
                        copies.append((used, whole[of[b], i], c - i * page))
                    else:
                        whole[of[b], i] = used
                used += 1
        order = torch.randperm(used + 2, generator=g)
        self.table = torch.where(table >= 0, order.to(torch.int32)[table.clamp(min=0).long()], table)
        self.k, self.v = (torch.randn(used + 2, self.Hkv, page, D, generator=g).to(dtype) for _ in range(2))
        for to, src, m in copies:
            for pool in (self.k, self.v):
                pool[order[to], :, :m] = pool[order[src], :, :m]
        self.q = torch.randn(self.rows, self.Hq, D, generator=g).to(dtype)
        self.cap = each * page
        self.n_cap = min(self.cap, max(self.n) + 30)

    def check(self, window=0, sink=0, scores=True, scale=None, start=None, common=None, groups=True, nan=(), finite_k=None):
        """nan: (sequence, kv head, query heads) whose logits have a NaN that the reference leaves out.  finite_k: keys by which
        a logit's rounding error is bounded where some are infinite (a logit of -Inf has none)."""
        d = kvr.make_desc(self.B, self.Hq, self.Hkv, 1, 1, self.dtype, softmax_scale=scale)
        i32 = lambda x: torch.tensor(x, dtype=torch.int32).cuda()
        pages = kvr.make_pages(d, self.k.cuda(), self.v.cuda(), self.table.cuda())
        grp = kvr.make_groups(i32(self.start if start is None else start), i32(self.common if common is None else common)) if groups else None
        old = torch.rand(self.B, self.Hkv, self.n_cap, generator=self.g) if scores else None
        sc = old.cuda() if scores else None
        out = torch.full((self.rows, self.Hq, D), 7.0, dtype=self.dtype).cuda()
        n = kvr.kvr_attend_shared_workspace_size(d, self.rows, pages, grp, window, sink, scores)
        ws = torch.randint(0, 256, (max(n, 256),), dtype=torch.uint8).cuda()
        qs = None if self.q_start is None else i32(self.q_start)
        kvr.kvr_attend_shared(d, self.q.cuda(), self.rows, qs, i32(self.n), pages, grp, window, sink, out, sc, self.n_cap if scores else 0, ws)
        torch.cuda.synchronize()
        ref = R.attend(self.q, self.k, self.v, self.table, self.n, self.q_start, d.softmax_scale, window, sink, self.n_cap, self.Hkv)
        if finite_k is not None:
            ref["e"] = R.attend(self.q, finite_k, self.v, self.table, self.n, self.q_start, d.softmax_scale, window, sink, self.n_cap, self.Hkv)["e"]
        for b, h, heads in nan:
            ref["out"][b, heads] = math.nan
            ref["scores"][b, h, :self.n[b]] = math.nan
        tol, tol_s = R.attend_bounds(ref, self.dtype, old)
        out = out.cpu()
        mine = ref["rows"]
        nan = ref["out"].isnan()
        assert torch.equal(out.isnan() & mine[:, None, None], nan & mine[:, None, None])
        err = (out.double() - ref["out"]).abs()
        fin = torch.isfinite(ref["out"]) & mine[:, None, None]
        assert bool((err <= tol)[fin].all()), float((err - tol)[fin].max())
        inf = torch.isinf(ref["out"]) & mine[:, None, None]
        assert torch.equal(out[inf].double(), ref["out"][inf])
        assert bool((out[~mine] == 7.0).all())
        if scores:
            grown = sc.cpu().double() - old.double()
            ok = (grown - ref["scores"]).abs() <= tol_s
            assert bool((ok | ref["scores"].isnan()).all()), float(((grown - ref["scores"]).abs() - tol_s).nan_to_num().max())
            assert torch.equal(grown.isnan(), ref["scores"].isnan())
        return out, sc


def one(*n):
    return [(x, 1) for x in n]


CASES = [  # groups, heads, page, lead, trail, alone, by q_start
    ([(1000, one(1001, 1040, 1500, 1000))], (32, 8), 16, 0, 0, (), False),           # the last has no token of its own
    ([(300, one(301, 420)), (0, one(70, 1)), (64, one(65, 64, 200))], (8, 2), 64, 0, 0, one(90, 0), False),
    ([(129, one(130, 0, 50, 700, 129))], (8, 8), 24, 0, 0, (), False),               # an empty row, and one that is shorter than what is shared
    ([(500, one(501)), (77, one(78, 79, 0))], (16, 2), 7, 0, 0, (), False),          # a group of one; pages of an odd size
    ([(200, [(210, 5), (200, 1), (333, 30), (201, 0)])], (32, 8), 32, 3, 2, [(40, 40)], True),
    ([(640, [(700, 8)] * 9)], (16, 2), 64, 0, 0, (), True),                          # 72 rows of 8 heads: several tiles of columns
    ([(640, [(700, 60)] * 9)], (16, 2), 64, 0, 0, (), True),                         # too many rows to share
    ([(250, [(260, 20), (251, 1), (900, 100)])], (2, 2), 1, 0, 5, (), True),          # the first has new rows among what is shared
    ([(64, one(65, 70, 64, 90, 128, 129)), (65, one(66, 67, 68, 69, 70)), (128, one(129, 130, 131))], (4, 2), 8, 0, 0, (), False),
    ([(200, [(203, 3), (210, 2), (201, 1), (264, 33)] * 3)], (4, 1), 16, 0, 0, (), True),      # 117 columns
    ([(300, one(*[301 + i for i in range(6)])), (300, one(*[310 + i for i in range(12)])), (300, one(*[301 + i for i in range(30)]))],
     (8, 2), 16, 0, 0, (), False),                                                   # 24, 48 and 120 columns
    ([(2048, one(*range(2049, 2100)))], (64, 8), 128, 0, 0, (), False),               # 408 columns
    ([(3000, one(*[3000 + 7 * i for i in range(1, 40)])), (100, one(101, 102))], (8, 1), 48, 0, 0, one(1, 2, 3), False),
]


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("case", range(len(CASES)))
def test_against_each_sequence_by_itself(case, dtype):
    groups, heads, page, lead, trail, alone, rows = CASES[case]
    b = Batch(groups, heads, page, dtype, 40 + case, lead=lead, trail=trail, alone=alone, rows=rows)
    b.check()
    b.check(scores=False)


def _many(rows, members, common):
    """A group, its sequences' own tokens from none (a sequence that is shorter than what it shares) to 300."""
    return common, [(max(common + 37 * i % 301 - (9 if i == 3 else 0), 0), 1 + i % rows) for i in range(members)]


WINDOWS = [  # rows of a sequence at most, groups, heads, page, window, first tokens: batches whose windows make a cache worth sharing
    (1, [_many(1, 40, 500), _many(1, 35, 129), _many(1, 30, 64), _many(1, 25, 1000)], (16, 8), 16, 400, 0),
    (1, [_many(1, 60, 450), _many(1, 66, 430)], (8, 8), 24, 390, 4),
    (1, [_many(1, 70, 640), _many(1, 30, 131)], (64, 8), 5, 500, 130),
    (1, [_many(1, 560, 70)], (8, 8), 16, 90, 3),
    (4, [_many(4, 40, 500), _many(4, 35, 129), _many(4, 30, 64), _many(4, 25, 1000)], (16, 8), 8, 260, 20),
    (9, [_many(9, 20, 900)], (4, 4), 64, 530, 3),
    (5, [_many(5, 60, 900), _many(5, 50, 640)], (8, 8), 16, 700, 9),
]


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("case", range(len(WINDOWS)))
def test_windows(case, dtype):
    """With pages that are not there, and values that are not finite where some columns see them and others do not."""
    most, groups, heads, page, window, sink = WINDOWS[case]
    b = Batch(groups, heads, page, dtype, 80 + case, rows=most > 1, room=0)
    b.check(window, sink)
    b.check(window, sink, scores=False)
    for i, (c, (first, end)) in enumerate(zip(b.common, zip(b.start, b.start[1:]))):
        if i % 2 == 0:                                           # a page of what is shared
            at = max(c - window, 0) // page + 1
            if (at + 1) * page <= c:
                b.table[first:end, at] = -1
        for j, what in ((c - 1, math.nan), (max(c - window + 100, 0), math.inf), (sink // 2, -math.inf)):
            for s in range(first, end):                          # (copies of a page that is filled in part have it too)
                at = R.token_row(b.k, b.table, s, j) if j < b.n[s] else None
                if at is not None:
                    b.v[at[0], 1, at[1], 64 + i] = what
        last = end - 1
        at = R.token_row(b.k, b.table, last, b.n[last] - 1)
        if at is not None:
            b.v[at[0], 0, at[1], 3] = math.inf
    b.check(window, sink)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("window,sink", [(0, 0), (600, 130), (33, 4), (1, 0), (1, 3)])
@pytest.mark.parametrize("case", range(len(CASES)))
def test_small_caches(case, window, sink, dtype):
    """Those that every sequence reads for itself."""
    groups, heads, page, lead, trail, alone, rows = CASES[case]
    b = Batch(groups, heads, page, dtype, 60 + case, lead=lead, trail=trail, alone=alone, rows=rows, room=0)
    b.check(window, sink)
    b.check(window, sink, scores=False)


@pytest.mark.parametrize("dtype", [BF, F32])
def test_no_groups_and_groups_that_share_nothing(dtype):
    b = Batch([(0, one(200, 31, 0, 900))], (8, 2), 16, dtype, 3, rows=False)
    none, sc0 = b.check(groups=False)
    for start, common in (([0, 4], [0]), ([0, 1, 2, 3, 4], [500, 31, 7, 2]), ([2, 2, 2], [9, 9]), ([4, 9], [8])):
        b.g.manual_seed(3)
        b.check(start=start, common=common)


@pytest.mark.parametrize("dtype", [BF, F32])
def test_starts_that_go_past_the_batch_and_more_in_common_than_there_is_room_for(dtype):
    b = Batch([(96, one(100, 120, 97, 98, 99, 96))], (8, 2), 32, dtype, 8, rows=False)
    b.check(start=[-5, 77], common=[96])
    b.check(start=[0, 6], common=[1 << 30])           # (more than each has: each by itself)
    b.check(start=[0, 6], common=[-4])
    b.check(start=[0, 1, 6], common=[96, 90])


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("page", [8, 64, 5])
def test_pages_that_are_not_there(dtype, page):
    """Among what is shared (for all alike) and among a sequence's own."""
    b = Batch([(320, one(400, 321, 500))], (8, 2), page, dtype, 12, rows=False)
    b.table[:, 1] = -1
    b.table[:, 192 // page] = 1 << 20
    b.table[0, 384 // page] = -7
    b.table[2, 448 // page:] = -1
    b.check()
    b.table[:, :320 // page] = -1                     # nothing of it
    b.check()


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("what", [math.inf, -math.inf, math.nan])
def test_values_that_are_not_finite(dtype, what):
    """Where no query sees them they do nothing; where one does they are its, not its neighbours'."""
    b = Batch([(320, [(350, 9), (323, 3), (540, 1)])], (8, 2), 16, dtype, 15)
    rows = [R.token_row(b.k, b.table, i, j) for i, j in ((0, 349), (0, 345), (2, 539), (2, 510))]
    shared = R.token_row(b.k, b.table, 0, 150)
    for page, row in rows + [shared]:
        b.v[page, 1, row, 5] = what
        b.v[page, 0, row, 127] = what
    # and tokens of nobody: behind the sequences' ends, and of pages that nobody names
    for i, n in enumerate(b.n):
        page, row = R.token_row(b.k, b.table, i, n - 1)
        b.k[page, :, row + 1:] = what
        b.v[page, :, row + 1:] = what
    named = set(b.table.flatten().tolist())
    for page in set(range(b.k.shape[0])) - named:
        b.k[page] = b.v[page] = what
    b.check()


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("where", ["shared", "own"])
def test_logits_that_are_not_finite(dtype, where):
    """NaN among the logits of one sequence's query, -Inf among all of another's."""
    b = Batch([(130, one(190, 131, 250, 140))], (4, 2), 16, dtype, 16, rows=False)
    page, row = R.token_row(b.k, b.table, 0, 100 if where == "shared" else 180)
    if where == "shared":
        b.q[0, 1, 3] = math.nan
        b.check(nan=[(0, 0, [1])])
    else:
        b.k[page, 1, row, 0] = math.nan
        b.check(nan=[(0, 1, [2, 3])])
    b2 = Batch([(130, one(190, 131, 250, 140))], (4, 2), 16, dtype, 17, rows=False)
    page, row = R.token_row(b2.k, b2.table, 0, 100 if where == "shared" else 180)
    b2.k[page, 1, row] = 0
    k0 = b2.k.clone()
    b2.k[page, 1, row, 0] = -math.inf
    b2.q[:, :, 0] = b2.q[:, :, 0].abs() + 1
    b2.check(finite_k=k0)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("scale", [0.0, -0.2, 3.0])
def test_scales(dtype, scale):
    Batch([(150, one(190, 151, 250, 152)), (33, one(40, 41))], (8, 2), 16, dtype, 18, rows=False).check(scale=scale)


@pytest.mark.parametrize("dtype", [BF, F32])
def test_a_first_token_that_draws_most_weight_and_logits_far_apart(dtype):
    """The maximum in what is shared for some heads, in a sequence's own for others."""
    b = Batch([(700, one(900, 701, 780))], (8, 2), 16, dtype, 19, rows=False)
    for h, (i, j) in enumerate(((0, 0), (0, 850))):
        page, row = R.token_row(b.k, b.table, i, j)
        b.k[page, h, row] = b.q[0, 4 * h] * 9
    b.check()


@pytest.mark.parametrize("dtype", [BF, F32])
def test_the_same_call_gives_the_same_bits(dtype):
    b = Batch([(1500, one(*range(1501, 1520))), (90, one(100, 91))], (8, 2), 16, dtype, 20, rows=False)
    got = []
    for _ in range(3):
        b.g.manual_seed(1)
        got.append(b.check())
    for out, sc in got[1:]:
        assert torch.equal(out, got[0][0]) and torch.equal(sc, got[0][1])


def test_a_place_for_fewer_scores_than_tokens():
    for dtype in (BF, F32):
        b = Batch([(300, one(400, 330))], (8, 2), 16, dtype, 21, rows=False)
        b.n_cap = 250
        b.check()
        b.n_cap = 310
        b.check()


@pytest.mark.parametrize("dtype,groups,heads", [
    (BF, [(30000, one(30100, 30001, 30500))], (8, 2)), (F32, [(9000, one(9100, 9001))], (4, 4)),
    (BF, [(20, one(*[21 + i % 50 for i in range(300)]))], (4, 1)), (F32, [(20, one(*[21 + i % 50 for i in range(150)]))], (4, 1)),
    (BF, [(5 + i, one(6 + i, 7 + i, 90)) for i in range(70)], (2, 2)), (BF, [(100 + i, one(*[101 + i + j for j in range(6)])) for i in range(150)], (2, 2))])
def test_long_ones_and_many(dtype, groups, heads):
    Batch(groups, heads, 16, dtype, 22, rows=False).check()


def _ends(members, common, most):
    """Sequences with ends of one token to `most` behind what they share, one without, one shorter, one empty."""
    n = [common + 1 + (i * i * 13 + 5 * i) % most for i in range(members)]
    n[1], n[2], n[3 % members] = common, max(common - 70, 0), 0
    n[4], n[5] = common + 256, common + 257                     # as many as the join takes, and one more
    return common, one(*n)


ENDS = [  # groups, heads, page, window, first tokens: sequences times kv heads from 512 on, whose last tokens the join attends to
    ([_ends(64, 500, 200)], (8, 8), 16, 0, 0),
    ([_ends(40, 640, 300), _ends(30, 64, 90)], (16, 8), 24, 0, 0),
    ([_ends(66, 300, 64)], (32, 8), 5, 0, 0),
    ([_ends(20, 1000, 256), _ends(49, 3, 300)], (64, 8), 64, 0, 0),
    ([_ends(64, 500, 300)], (32, 8), 16, 150, 5),
    ([_ends(70, 200, 300)], (8, 8), 7, 30, 230),
    ([_ends(64, 900, 300)], (32, 8), 16, 700, 5),
    ([_ends(70, 450, 300)], (8, 8), 7, 300, 500),
]


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("case", range(len(ENDS)))
def test_many_sequences_with_short_ends(case, dtype):
    """Also with pages that are not there, values that are not finite, and fewer scores than tokens."""
    groups, heads, page, window, sink = ENDS[case]
    b = Batch(groups, heads, page, dtype, 90 + case, rows=False, room=20000 if window == 0 else 30000)
    out, sc = b.check(window, sink)
    b.g.manual_seed(90)
    first = b.check(window, sink)
    b.g.manual_seed(90)
    again = b.check(window, sink)
    assert all(torch.equal(x, y) for x, y in zip(first, again))
    b.check(window, sink, scores=False)
    for s in range(6, 20, 3):                                    # pages behind what is shared
        last = (b.n[s] - 1) // page
        if last * page >= groups[0][0]:
            b.table[s, last] = -1 if s % 2 else 1 << 20
    for s, what in ((7, math.inf), (8, math.nan), (10, -math.inf)):
        at = R.token_row(b.v, b.table, s, b.n[s] - 1)
        if at is not None and b.n[s] > groups[0][0]:
            b.v[at[0], 2, at[1], 77] = what
            if b.n[s] % page:                                    # and behind its end
                b.k[at[0], :, b.n[s] % page:] = math.nan
                b.v[at[0], :, b.n[s] % page:] = math.nan
    b.n_cap = groups[0][0] + 40
    b.check(window, sink)


@pytest.mark.parametrize("dtype", [BF, F32])
def test_logits_that_are_not_finite_among_many_short_ends(dtype):
    """NaN in one sequence's query, in a key of another's end, and -Inf as the only logits of a third (one token of its own, no group)."""
    b = Batch([_ends(64, 200, 150)], (16, 8), 16, dtype, 97, alone=one(1, 40), rows=False, room=20000)
    b.q[9, 5, 3] = math.nan
    page, row = R.token_row(b.k, b.table, 12, b.n[12] - 1)
    b.k[page, 3, row, 0] = math.nan
    page, row = R.token_row(b.k, b.table, 64, 0)
    b.k[page, 1, row] = 0
    k0 = b.k.clone()
    b.k[page, 1, row, 0] = -math.inf
    b.q[64, 2:4, 0] = b.q[64, 2:4, 0].abs() + 1
    k0 = torch.nan_to_num(k0)
    b.check(nan=[(9, 2, [5]), (12, 3, [6, 7])], finite_k=k0)

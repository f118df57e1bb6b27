"""Caches with room for far more tokens than their sequences have: results do not depend on the room, and the largest sizes that
the calls accept are launched."""
import pytest
import torch

from paper_2512_17917_amd import binding as kvr
from tests import cache_ref as R
from tests.test_gpu_cache_ops import _attend, _cache, _dev, _normal, _starts

pytestmark = [pytest.mark.gpu, pytest.mark.timeout(300)]
D = 128
BF, F32 = torch.bfloat16, torch.float32


ROOMY = [  # which, dtype, heads, page, lengths, new, window, sinks, n_cap (0: all there is room for), room
    ("prompt", BF, (32, 8), 16, [200], [200], 0, 0, 0, 131072),
    ("prompt", BF, (8, 2), 64, [700, 0, 300, 41], [700, 0, 290, 1], 0, 0, 0, 32768),
    ("prompt", BF, (8, 8), 24, [520, 600], [7, 600], 0, 0, 550, 24000),
    ("prompt", BF, (4, 2), 16, [1500, 900], [1500, 20], 300, 40, 0, 65536),
    ("prompt", BF, (8, 1), 16, [2600], [130], 400, 3, 2300, 40000),
    ("prompt", BF, (16, 2), 1, [300, 5], [290, 5], 0, 0, 0, 5000),
    ("prompt", BF, (2, 2), 16, [30 + b for b in range(70)], [b % 5 for b in range(70)], 0, 0, 0, 16384),
    ("prompt", F32, (8, 2), 16, [333, 0, 70], [333, 0, 9], 0, 0, 0, 131072),
    ("prompt", F32, (4, 4), 24, [500], [500], 100, 20, 450, 48000),
    ("paged", BF, (32, 8), 16, [1000, 1, 0], None, 0, 0, 0, 131072),
    ("paged", BF, (8, 2), 16, [(37 * b) % 900 for b in range(40)], None, 0, 0, 0, 32768),
    ("paged", F32, (16, 2), 24, [700, 33], None, 100, 16, 0, 48000),
]


@pytest.mark.parametrize("case", range(len(ROOMY)))
def test_room_does_not_change_results(case):
    which, dtype, (Hq, Hkv), page, n, new, window, sink, n_cap, room = ROOMY[case]
    g = torch.Generator().manual_seed(600 + case)
    B, most = len(n), max(n)
    q_start = None if new is None else _starts(new, 1)
    rows = B if new is None else q_start[-1] + 2
    kp, vp, table = _cache(g, B, Hkv, most, page, dtype)
    wide = torch.full((B, room // page), -1, dtype=torch.int32)
    wide[:, :table.shape[1]] = table
    q = _normal(g, rows, Hq, D, dtype=dtype)
    d = kvr.make_desc(B, Hq, Hkv, 1, 1, dtype)
    q_d, kp_d, vp_d, wide_d = _dev(q, kp, vp, wide)
    qs = None if q_start is None else torch.tensor(q_start, dtype=torch.int32).cuda()
    nc = torch.tensor(n, dtype=torch.int32).cuda()
    pages = kvr.make_pages(d, kp_d, vp_d, wide_d)
    n_cap = n_cap or room
    old = torch.rand(B, Hkv, n_cap, generator=g)
    sc = old.cuda()
    out = _attend(which, d, q_d, rows, qs, nc, pages, window, sink, sc, n_cap).cpu()
    ref = R.attend(q, kp, vp, table, n, q_start, d.softmax_scale, window, sink, n_cap, Hkv)
    tol, tol_s = R.attend_bounds(ref, dtype, old)
    mine = ref["rows"]
    assert bool(((out.double() - ref["out"]).abs() <= tol)[mine].all()) and bool((out[~mine] == 7.0).all())
    err = (sc.cpu().double() - old.double() - ref["scores"]).abs()
    assert bool((err <= tol_s).all()), (float(err.max()), (err > tol_s).nonzero()[:4].tolist())
    assert torch.equal(sc.cpu()[ref["scores"] == 0], old[ref["scores"] == 0])
    again = old.cuda()
    _attend(which, d, q_d, rows, qs, nc, pages, window, sink, again, n_cap, ws_fill=0)
    assert torch.equal(again, sc)


def _shared(g, heads, page, dtype):
    """One page that every entry of a table names, so that a small pool makes a long cache."""
    kp, vp = (_normal(g, 1, heads, page, D, dtype=dtype) for _ in range(2))
    return kp, vp


def _large(dtype, B, H, page, room, n, new, seed):
    """A prompt's call on a cache of `room` tokens a sequence, scores for all of them; -> error over bound, for the tokens there are."""
    g = torch.Generator().manual_seed(seed)
    kp, vp = _shared(g, H, page, dtype)
    q_start = _starts(new)
    rows = q_start[-1]
    q = _normal(g, rows, H, D, dtype=dtype)
    d = kvr.make_desc(B, H, H, 1, 1, dtype)
    table = torch.zeros(B, room // page, dtype=torch.int32, device="cuda")
    q_d, kp_d, vp_d = _dev(q, kp, vp)
    pages = kvr.make_pages(d, kp_d, vp_d, table)
    sc = torch.zeros(B, H, room, device="cuda")
    out = _attend("prompt", d, q_d, rows, torch.tensor(q_start, dtype=torch.int32).cuda(), torch.tensor(n, dtype=torch.int32).cuda(), pages,
                  0, 0, sc, room).cpu()
    most = max(n)
    few = torch.zeros(B, -(-most // page), dtype=torch.int32)
    ref = R.attend(q, kp, vp, few, n, q_start, d.softmax_scale, 0, 0, most, H)
    tol, tol_s = R.attend_bounds(ref, dtype)
    assert bool(((out.double() - ref["out"]).abs() <= tol).all())
    assert bool(((sc[:, :, :most].cpu().double() - ref["scores"]).abs() <= tol_s).all())
    assert not any(bool(sc[b, :, most:].any()) for b in range(B))


def test_scores_of_four_billion_tokens_of_room():
    """512 sequences of 8 heads with room for 2^20 tokens each: 2^32 scores, 17 GB."""
    n, new = [0] * 512, [0] * 512
    for b, x, y in ((0, 300, 300), (3, 700, 4), (511, 280, 33)):
        n[b], new[b] = x, y
    _large(BF, 512, 8, 4096, 1 << 20, n, new, 1)


def test_scores_of_more_blocks_than_a_launch_has():
    """8192 heads whose longest sequences have three blocks of tokens: the last ones lie beyond the launch's 16384 workgroups."""
    n, new = [0] * 1024, [0] * 1024
    for b, x, y in ((0, 700, 700), (1, 100, 100), (500, 650, 3), (1023, 513, 40)):
        n[b], new[b] = x, y
    _large(BF, 1024, 8, 64, 1024, n, new, 3)


@pytest.mark.parametrize("room", [1 << 28, (1 << 28) + (1 << 20)])
def test_scores_of_one_long_room_float32(room):
    """2^28 tokens of room for one head, and more."""
    _large(F32, 1, 1, 1 << 16, room, [777], [130], 2)


def test_rotation_of_more_rows_than_a_launch_has_waves():
    """2^26 + 5 rows (17 GB of keys, in place): the last ones as a call on them alone gives them."""
    n = (1 << 26) + 5
    d = kvr.make_desc(1, 1, 1, 1, 1, BF)
    inv = (1e4 ** (-torch.arange(64, dtype=torch.float64) / 64)).cuda()
    turn = kvr.make_rotation(d, inv)
    k = torch.zeros(n, 1, D, dtype=BF, device="cuda")
    some = torch.randn(9, 1, D, generator=torch.Generator().manual_seed(1)).to(BF).cuda()
    k[:9], k[-9:] = some, some
    nc = torch.tensor([n], dtype=torch.int32).cuda()
    want = []
    for end in (9, n):
        alone = some.clone()
        kvr.kvr_rotate(d, turn, None, alone, None, 9, torch.tensor([0, 9], dtype=torch.int32).cuda(),
                       torch.tensor([end], dtype=torch.int32).cuda(), None, alone)
        want.append(alone)
    kvr.kvr_rotate(d, turn, None, k, None, n, torch.tensor([0, n], dtype=torch.int32).cuda(), nc, None, k)
    assert torch.equal(k[:9], want[0]) and torch.equal(k[-9:], want[1])
    assert not torch.equal(want[0], some)

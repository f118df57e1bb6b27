"""kvr_rotate_axes against float64, and against kvr_rotate where all axes count tokens."""
import pytest
import torch

from paper_2512_17917_amd import binding as kvr
from tests import cache_ref as R
from tests.test_gpu_cache_ops import _cache, _dev, _normal, _starts

pytestmark = [pytest.mark.gpu, pytest.mark.timeout(300)]
D = 128
BF, F32 = torch.bfloat16, torch.float32


def _turned(x, w, pos, axis, inv, eps, pairs):
    """As R.rotate, pair by pair: the position of its axis."""
    y, size = R.rotate(x, w, torch.zeros(x.shape[0]), None, eps, pairs)
    y, size = y.clone(), size.clone()
    n = len(axis)
    for i in range(n):
        lo, hi = (2 * i, 2 * i + 1) if pairs else (i, i + n)
        a = (pos[axis[i]].double() * inv[i])[:, None]
        u, v = y[..., lo].clone(), y[..., hi].clone()
        y[..., lo], y[..., hi] = u * a.cos() - v * a.sin(), v * a.cos() + u * a.sin()
        size[..., lo] = size[..., hi] = u.abs() + v.abs()
    return y, size


CASES = [  # dtype, heads, rot, pairs, norm, page, tokens, new (None: one row a sequence), first row, axes, spread of positions
    (BF, (32, 8), 128, False, True, 64, [32768], None, 0, 3, 1 << 20),
    (BF, (8, 2), 128, False, True, 16, [200, 0, 77], [200, 0, 5], 0, 3, 300),
    (BF, (8, 8), 64, True, True, 24, [31, 1, 130], [31, 1, 100], 3, 2, 5000),
    (BF, (64, 8), 32, False, False, 100, [129], [129], 0, 8, 1 << 30),
    (BF, (4, 4), 20, False, True, 7, [40, 13], [33, 13], 1, 5, 40),          # pairs that share no lane layout
    (BF, (16, 8), 2, False, True, 5, [9, 70], [9, 70], 0, 1, 100),
    (F32, (16, 8), 128, False, True, 16, [333, 1, 0, 12], [333, 1, 0, 12], 0, 3, 1000),
    (F32, (16, 16), 32, True, False, 0, [57, 57], [57, 20], 2, 2, 60),
    (F32, (1, 1), 126, False, True, 1, [3, 300], [3, 300], 0, 4, 300),
    (F32, (8, 2), 8, False, True, 48, [2083, 2], None, 0, 4, 2083),
]


@pytest.mark.parametrize("case", range(len(CASES)))
def test_axes(case):
    dtype, (Hq, Hkv), rot, pairs, norm, page, n_ctx, new, lead, n_axes, spread = CASES[case]
    g = torch.Generator().manual_seed(300 + case)
    B, half = len(n_ctx), rot // 2
    q_start = None if new is None else _starts(new, lead)
    rows = B if new is None else q_start[-1] + 2                         # and two rows of nobody
    kp, vp, table = _cache(g, B, Hkv, max(max(n_ctx), 1), page, dtype)
    fused = _normal(g, rows, Hq + 2 * Hkv, D, dtype=dtype)
    q, k, v = fused[:, :Hq], fused[:, Hq:Hq + Hkv], fused[:, Hq + Hkv:]
    wq, wk = ((_normal(g, D, dtype=F32) * 0.3 + 1).to(dtype) for _ in range(2)) if norm else (None, None)
    inv = 1e6 ** (-torch.arange(half, dtype=torch.float64) / half)
    axis = torch.randint(n_axes, (half,), generator=g).tolist()
    pos = torch.randint(-spread, spread + 1, (n_axes, rows + 3), generator=g, dtype=torch.int32)     # rows of an axis further apart
    d = kvr.make_desc(B, Hq, Hkv, 1, 1, dtype)
    f_d, kp_d, vp_d, table_d, wq_d, wk_d, inv_d, pos_d = _dev(fused, kp, vp, table, wq, wk, inv, pos)
    pages = kvr.make_pages(d, kp_d, vp_d, table_d)
    turn = kvr.make_rotation(d, inv_d, q_weight=wq_d, k_weight=wk_d, eps=1e-6, pairs=pairs)
    q_out, k_out = torch.full((rows, Hq, D), 7.0, dtype=dtype).cuda(), torch.full((rows, Hkv, D), 7.0, dtype=dtype).cuda()
    qs = None if q_start is None else torch.tensor(q_start, dtype=torch.int32).cuda()
    nc = torch.tensor(n_ctx, dtype=torch.int32).cuda()
    kvr.kvr_rotate_axes(d, turn, kvr.make_axes(axis, n_axes), pos_d, f_d[:, :Hq], f_d[:, Hq:Hq + Hkv], f_d[:, Hq + Hkv:], rows, qs, nc,
                        q_out, k_out, pages)
    torch.cuda.synchronize()
    mine = torch.zeros(rows, dtype=torch.bool)
    kp0, vp0, stored = kp.clone(), vp.clone(), {}
    for b, (r0, y) in enumerate(R.spans(B, rows, q_start)):
        mine[r0:r0 + y] = True
        for r in range(r0, r0 + y):
            j = n_ctx[b] - y + r - r0
            if 0 <= j < R.capacity(kp, table):
                stored[R.token_row(kp, table, b, j)] = r
    for x, w, got in ((q, wq, q_out), (k, wk, k_out)):
        ref, size = _turned(x, w, pos[:, :rows], axis, inv, 1e-6, pairs)
        err = (got.cpu().double() - ref).abs()
        assert bool((err <= R.rotate_bound(ref, size, dtype))[mine].all()), float(err[mine].max())
        assert bool((got.cpu()[~mine] == 7.0).all())
    ko = k_out.cpu()
    for (page_i, row), r in stored.items():
        kp0[page_i, :, row], vp0[page_i, :, row] = ko[r], v[r]
    assert torch.equal(kp_d.cpu(), kp0) and torch.equal(vp_d.cpu(), vp0)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("rot,pairs", [(128, False), (64, True), (32, False), (12, False)])
def test_positions_that_count_tokens_make_what_rotate_makes(dtype, rot, pairs):
    """Bit for bit; one row of positions for all axes (stride 0) and a row each."""
    g = torch.Generator().manual_seed(9)
    n_ctx, new = [70, 33, 5], [20, 33, 1]
    q_start = _starts(new)
    rows, Hq, Hkv = q_start[-1], 8, 2
    d = kvr.make_desc(3, Hq, Hkv, 1, 1, dtype)
    q, k = _normal(g, rows, Hq, D, dtype=dtype).cuda(), _normal(g, rows, Hkv, D, dtype=dtype).cuda()
    inv = (1e6 ** (-torch.arange(rot // 2, dtype=torch.float64) / (rot // 2))).cuda()
    turn = kvr.make_rotation(d, inv, pairs=pairs, q_weight=_normal(g, D, dtype=dtype).cuda())
    nc, qs = torch.tensor(n_ctx, dtype=torch.int32).cuda(), torch.tensor(q_start, dtype=torch.int32).cuda()
    want = torch.empty_like(q), torch.empty_like(k)
    kvr.kvr_rotate(d, turn, q, k, None, rows, qs, nc, *want)
    one = torch.cat([torch.arange(n - y, n) for n, y in zip(n_ctx, new)]).to(torch.int32).cuda()
    axes = kvr.make_axes([i % 3 for i in range(rot // 2)])
    for pos in (one[None].expand(3, rows), one[None].repeat(3, 1)):
        got = torch.empty_like(q), torch.empty_like(k)
        kvr.kvr_rotate_axes(d, turn, axes, pos, q, k, None, rows, qs, nc, *got)
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


@pytest.mark.parametrize("dtype,rows", [(BF, 1), (BF, 777), (F32, 130)])
def test_rows_of_no_sequence(dtype, rows):
    """Without a cache: any number of rows, in place, no lengths; and nothing turned at all, without positions."""
    g = torch.Generator().manual_seed(rows)
    Hq, Hkv = 4, 4
    d = kvr.make_desc(2, Hq, Hkv, 1, 1, dtype)
    q, k = _normal(g, rows, Hq, D, dtype=dtype), _normal(g, rows, Hkv, D, dtype=dtype)
    inv = 1e4 ** (-torch.arange(32, dtype=torch.float64) / 32)
    axis = [i // 16 for i in range(32)]
    pos = torch.randint(0, 90, (2, rows), generator=g, dtype=torch.int32)
    turn = kvr.make_rotation(d, inv.cuda(), pairs=True)
    qd, kd = q.cuda(), k.cuda()
    kvr.kvr_rotate_axes(d, turn, kvr.make_axes(axis), pos.cuda(), qd, kd, None, rows, None, None, qd, kd)
    for x, got in ((q, qd), (k, kd)):
        ref, size = _turned(x, None, pos, axis, inv, 0, True)
        assert bool(((got.cpu().double() - ref).abs() <= R.rotate_bound(ref, size, dtype)).all())
    out = torch.empty_like(qd)
    kvr.kvr_rotate_axes(d, kvr.make_rotation(d), kvr.make_axes([]), None, qd, None, None, rows, None, None, out)
    assert torch.equal(out, qd)


def test_a_captured_call_follows_the_positions():
    g = torch.Generator().manual_seed(1)
    B, Hq, Hkv = 3, 8, 2
    d = kvr.make_desc(B, Hq, Hkv, 1, 1, BF)
    q, k, v = (_normal(g, B, h, D, dtype=BF).cuda() for h in (Hq, Hkv, Hkv))
    inv = (1e6 ** (-torch.arange(64, dtype=torch.float64) / 64)).cuda()
    turn, axes = kvr.make_rotation(d, inv), kvr.make_axes([i // 24 for i in range(64)])
    pos, nc = torch.zeros(3, B, dtype=torch.int32).cuda(), torch.zeros(B, dtype=torch.int32).cuda()
    table = torch.arange(6, dtype=torch.int32).view(3, 2).cuda()

    def call(pools, out):
        kvr.kvr_rotate_axes(d, turn, axes, pos, q, k, v, B, None, nc, out, None, kvr.make_pages(d, *pools, table))

    def pools():
        return [torch.zeros(6, Hkv, 16, D, dtype=BF).cuda() for _ in range(2)]

    held, out = pools(), torch.empty_like(q)
    call(held, out)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(held, out)
    for seed in range(4):
        pos.copy_(torch.randint(0, 5000, (3, B), generator=g, dtype=torch.int32))
        nc.copy_(torch.tensor([seed, 32 - seed, 17 + seed], dtype=torch.int32))
        for x in held:
            x.zero_()
        graph.replay()
        torch.cuda.synchronize()
        fresh, want = pools(), torch.empty_like(q)
        call(fresh, want)
        assert torch.equal(out, want) and torch.equal(held[0], fresh[0]) and torch.equal(held[1], fresh[1])

"""Rotation by positions on several axes and attention of groups that share their beginning run together, as PagedCache runs them: a
picture and its question prefilled once, sequences that begin with it, decode steps and drafts behind it, a captured step whose lengths
and groups change between replays, and calls on two streams at once."""
import pytest
import torch

from paper_2512_17917_amd import binding as kvr
from paper_2512_17917_amd.state import LayerState, PagedCache
from tests import cache_ref as R
from tests.test_gpu_cache_state import _near, _rotation
from tests.test_gpu_shared import ROOM

pytestmark = [pytest.mark.gpu, pytest.mark.timeout(300)]
D = 128
BF, F32 = torch.bfloat16, torch.float32
AXIS = [i % 3 for i in range(60)] + [0] * 4


def _positions(text, rows, cols):
    """[3, n] of text tokens, a picture's rows x cols patches and one token more, and the position that follows."""
    t = torch.arange(text)
    pic = torch.stack([torch.full((rows * cols,), text), text + torch.arange(rows).repeat_interleave(cols), text + torch.arange(cols).repeat(rows)])
    after = text + max(rows, cols)
    return torch.cat([t.expand(3, -1), pic, torch.full((3, 1), after)], 1).to(torch.int32), after + 1


def _turn_ref(inv, x, w, pos, dtype):
    """R.rotate by three axes: the pairs of each axis by its positions."""
    y = x.double()
    if w is not None:
        y = y / (y.pow(2).mean(-1, keepdim=True) + 1e-6).sqrt() * w.double()
    a = torch.stack([pos[AXIS[i]].double() * inv[i] for i in range(64)], 1)[:, None]
    u, v = y[..., :64], y[..., 64:]
    return torch.cat([u * a.cos() - v * a.sin(), v * a.cos() + u * a.sin()], -1), torch.cat([u.abs() + v.abs()] * 2, -1)


@pytest.mark.parametrize("dtype,window,n_sink,room", [(BF, 0, 0, ROOM), (BF, 0, 0, 300), (BF, 90, 5, ROOM), (F32, 0, 0, ROOM)])
def test_a_picture_that_several_sequences_begin_with(dtype, window, n_sink, room):
    """Every stage against float64 of what the stage before it left on the GPU."""
    g = torch.Generator().manual_seed(11)
    B, Hq, Hkv, ps = 5, 8, 2, 16
    d = kvr.make_desc(B, Hq, Hkv, 1, 1, dtype)
    inv = 1e6 ** (-torch.arange(64, dtype=torch.float64) / 64)
    turn, _, wq, wk = _rotation(d, dtype, g)
    cols = -(-room // ps)
    c = PagedCache(d, n_pages=120, page_size=ps, table_cap=cols, rotation=turn, window=window, n_sink=n_sink, axes=kvr.make_axes(AXIS))
    free = torch.randperm(120, generator=g).tolist()
    take = lambda n: [free.pop() for _ in range(n)]
    pos, after = _positions(20, 13, 18)
    n0 = pos.shape[1]                                            # 255 tokens: the last page is filled in part
    c.assign(0, 0, take(16))
    q_start = [0] + [n0] * B
    x = torch.randn(n0, Hq + 2 * Hkv, D, generator=g).to(dtype)
    part = lambda t: (t[:, :Hq], t[:, Hq:Hq + Hkv], t[:, Hq + Hkv:])
    i32 = lambda t: torch.tensor(t, dtype=torch.int32).cuda()
    c.n_ctx.copy_(i32([n0] + [0] * (B - 1)))
    out = c.prompt(*part(x.cuda()), i32(q_start), pos=pos.cuda())
    k_ref, k_size = _turn_ref(inv, x[:, Hq:Hq + Hkv], wk, pos, dtype)
    q_ref, q_size = _turn_ref(inv, x[:, :Hq], wq, pos, dtype)
    kp, vp, table = c.k.cpu(), c.v.cpu(), c.table.cpu()
    for t in range(n0):
        page, row = R.token_row(kp, table, 0, t)
        assert bool(((kp[page, :, row].double() - k_ref[t]).abs() <= R.rotate_bound(k_ref[t], k_size[t], dtype)).all())
        assert torch.equal(vp[page, :, row], x[t, Hq + Hkv:])
    turned = torch.empty(n0, Hq, D, dtype=dtype).cuda()
    kvr.kvr_rotate_axes(d, turn, c.axes, pos.cuda(), x.cuda()[:, :Hq], None, None, n0, None, None, turned)
    assert bool(((turned.cpu().double() - q_ref).abs() <= R.rotate_bound(q_ref, q_size, dtype)).all())
    lens = [n0] + [0] * (B - 1)
    n_cap = min(c.n_cap, 400)
    ref = R.attend(turned.cpu(), kp, vp, table, lens, q_start, d.softmax_scale, window, n_sink, n_cap, Hkv)
    tol = _near(out, ref, dtype)
    assert bool(((c.scores[:, :, :n_cap].cpu().double() - ref["scores"]).abs() <= tol).all())

    for b in range(1, 4):                                        # three more that begin with it; the last of the batch is of no group
        c.begin_with(b, 0, n0, page=take(1)[0])
    assert torch.equal(c.scores[1], c.scores[0])
    for b in range(4):
        c.assign(b, 16, take(2))
    c.assign(4, 0, take(3))
    lens = [n0] * 4 + [0]
    c.n_ctx.copy_(i32(lens))
    c.share([0, 4], [n0])
    table = c.table.cpu()
    for step in range(4):
        before = c.scores[:, :, :n_cap].cpu()
        if step % 2 == 0:                                        # a question or draft: several tokens a sequence
            new = [3, 1, 6, 2, 40 if step == 0 else 0]
            starts = [0]
            for y in new:
                starts.append(starts[-1] + y)
        else:
            new, starts = [1] * B, None
        lens = [n + y for n, y in zip(lens, new)]
        at = torch.cat([torch.arange(n - y, n) - (n0 - after if b < 4 else 0) for b, (n, y) in enumerate(zip(lens, new))]).to(torch.int32)
        p = at.expand(3, -1).cuda()
        x = torch.randn(sum(new), Hq + 2 * Hkv, D, generator=g).to(dtype).cuda()
        if starts is None:
            out = c.decode_step(*part(x), pos=p)
            q = c.q
        else:
            c.n_ctx.copy_(i32(lens))
            out = c.prompt(*part(x), i32(starts), pos=p)
            q = torch.empty(sum(new), Hq, D, dtype=dtype).cuda()
            kvr.kvr_rotate_axes(d, turn, c.axes, p, x[:, :Hq], None, None, sum(new), None, None, q)
        kp, vp = c.k.cpu(), c.v.cpu()
        ref = R.attend(q.cpu(), kp, vp, table, lens, starts, d.softmax_scale, window, n_sink, n_cap, Hkv)
        tol = _near(out, ref, dtype, before)
        assert bool(((c.scores[:, :, :n_cap].cpu().double() - before.double() - ref["scores"]).abs() <= tol).all())
        assert c.n_ctx.tolist() == lens
    c.share(None, None)                                          # each by itself again
    lens = [n + 1 for n in lens]
    x = torch.randn(B, Hq + 2 * Hkv, D, generator=g).to(dtype).cuda()
    out = c.decode_step(*part(x), pos=i32([lens] * 3))
    _near(out, R.attend(c.q.cpu(), c.k.cpu(), c.v.cpu(), table, lens, None, d.softmax_scale, window, n_sink, n_cap, Hkv), dtype)


@pytest.mark.parametrize("dtype", [BF, F32])
def test_a_compressed_layer_goes_on_by_axes(dtype):
    """LayerState.decode_step with positions on several axes: the key and query of kvr_rotate_axes, then the step with them."""
    g = torch.Generator().manual_seed(12)
    B, Hq, Hkv, N = 2, 8, 2, 90
    d = kvr.make_desc(B, Hq, Hkv, 3, 16, dtype, seed=3)
    inv = 1e6 ** (-torch.arange(64, dtype=torch.float64) / 64)
    turn, _, wq, wk = _rotation(d, dtype, g)
    K, V = (torch.randn(B, Hkv, N, D, generator=g).to(dtype) for _ in range(2))
    ls, _ = LayerState.from_prefill(d, K.cuda(), V.cuda(), torch.zeros(B, Hq, D, dtype=dtype).cuda(), n_recent=N, k_candidate=10, max_new_tokens=4)
    x = torch.randn(B, Hq + 2 * Hkv, D, generator=g).to(dtype)
    pos = torch.tensor([[40, 7], [41, 9], [50, 8]], dtype=torch.int32)
    xd = x.cuda()
    out = ls.decode_step(xd[:, Hq:Hq + Hkv], xd[:, Hq + Hkv:].contiguous(), xd[:, :Hq], rotation=turn, axes=kvr.make_axes(AXIS), pos=pos.cuda())
    qt, kt = ls.q_turned.cpu(), ls.k_turned.cpu()
    for got, part, w in ((qt, x[:, :Hq], wq), (kt, x[:, Hq:Hq + Hkv], wk)):
        ref, size = _turn_ref(inv, part, w, pos, dtype)
        assert bool(((got.double() - ref).abs() <= R.rotate_bound(ref, size, dtype)).all())
    K1, V1 = torch.cat([K, kt[:, :, None]], 2), torch.cat([V, x[:, Hq + Hkv:, None]], 2)
    _near(out, R.attend(qt, K1, V1, None, [N + 1] * B, None, d.softmax_scale, 0, 0, N + 4, Hkv), dtype)


# ---------------------------------------------------------------------------
B_, HQ, HKV, PAGE, POOL = 6, 8, 2, 16, 900
STEPS = [  # tokens of the sequences, groups' starts (four groups at most), tokens in common, new rows where there are starts
    ([3001, 3040, 3500, 3001, 700, 650], [0, 4, 6, 6, 6], [3000, 640, 0, 0], [1, 2, 3, 1, 5, 9]),
    ([3001, 3041, 3500, 3002, 0, 1], [0, 4, 6, 6, 6], [3000, 640, 0, 0], [1, 2, 3, 1, 0, 1]),
    ([900, 800, 700, 690, 680, 641], [0, 1, 2, 4, 6], [500, 500, 600, 640], [0, 0, 20, 0, 0, 1]),
    ([0] * 6, [0, 6, 6, 6, 6], [3000, 0, 0, 0], [1] * 6),
    ([3500] * 6, [0, 0, 0, 4, 6], [9, 9, 3000, 640], [16, 0, 1, 3, 2, 8]),
    ([3001, 3040, 3500, 3001, 700, 650], [0, 4, 6, 6, 6], [3000, 640, 0, 0], [1, 2, 3, 1, 5, 9]),
]


class _Call:
    def __init__(self, dtype, rows, window, sink, seed):
        """Sequences 0 .. 3 have their first 3000 tokens on the same pages, 4 and 5 their first 640; beyond them page numbers
        are drawn from the pool as they come (what they hold does not matter to results that are compared with each other)."""
        g = torch.Generator().manual_seed(seed)
        self.rows, self.window, self.sink = rows, window, sink
        self.d = kvr.make_desc(B_, HQ, HKV, 1, 1, dtype)
        self.k, self.v = (torch.randn(POOL, HKV, PAGE, D, generator=g).to(dtype).cuda() for _ in range(2))
        table = torch.full((B_, (4000 + ROOM) // PAGE), -1, dtype=torch.int32)
        table[:, :250] = torch.randint(0, POOL, (B_, 250), generator=g)
        table[:4, :188] = table[0, :188]
        table[4:, :40] = table[4, :40]
        self.table = table.cuda()
        self.pages = kvr.make_pages(self.d, self.k, self.v, self.table)
        self.n_rows = 40 if rows else B_
        self.q = torch.randn(self.n_rows, HQ, D, generator=g).to(dtype).cuda()
        self.out = torch.empty_like(self.q)
        self.scores = torch.empty(B_, HKV, 4000, device="cuda")
        i32 = lambda n: torch.zeros(n, dtype=torch.int32, device="cuda")
        self.n_ctx, self.q_start, self.start, self.common = i32(B_), i32(B_ + 1), i32(5), i32(4)
        self.groups = kvr.make_groups(self.start, self.common)
        n = kvr.kvr_attend_shared_workspace_size(self.d, self.n_rows, self.pages, self.groups, window, sink, True)
        self.ws = torch.empty(n, dtype=torch.uint8, device="cuda")

    def set(self, n, start, common, new):
        starts = [0]
        for y in new:
            starts.append(starts[-1] + y)
        for to, x in ((self.n_ctx, n), (self.q_start, starts), (self.start, start), (self.common, common)):
            to.copy_(torch.tensor(x, dtype=torch.int32))
        self.out.fill_(3.0)
        self.scores.fill_(0.5)

    def run(self):
        kvr.kvr_attend_shared(self.d, self.q, self.n_rows, self.q_start if self.rows else None, self.n_ctx, self.pages, self.groups, self.window,
                              self.sink, self.out, self.scores, 4000, self.ws)

    def results(self):
        return self.out.clone(), self.scores.clone()


@pytest.mark.parametrize("window,sink", [(0, 0), (300, 20)])
@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("rows", [False, True])
def test_a_captured_call_follows_lengths_and_groups(rows, dtype, window, sink):
    c = _Call(dtype, rows, window, sink, 31)
    graph = torch.cuda.CUDAGraph()
    c.set(*STEPS[0])
    with torch.cuda.graph(graph):                                # (for some of the cases the kernels' first call)
        c.run()
    want = []
    for s in STEPS:
        c.set(*s)
        c.ws.fill_(255)
        c.run()
        want.append(c.results())
    assert torch.equal(want[0][0], want[-1][0]) and torch.equal(want[0][1], want[-1][1])
    for s, (out, scores) in zip(STEPS, want):
        c.set(*s)
        c.ws.random_(0, 255)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(c.out, out) and torch.equal(c.scores, scores), s
        _ = (c.out.float() @ c.out.float().transpose(1, 2)).sum().item()


@pytest.mark.parametrize("dtype", [BF, F32])
def test_calls_on_two_streams_at_once(dtype):
    """Each with a workspace and results of its own, over the same cache."""
    a, b = _Call(dtype, False, 0, 0, 32), _Call(dtype, True, 0, 0, 32)
    b.k, b.v, b.table, b.pages = a.k, a.v, a.table, a.pages
    for c, s in ((a, STEPS[0]), (b, STEPS[4])):
        c.set(*s)
        c.run()
    want = [c.results() for c in (a, b)]
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for _ in range(5):
        for c in (a, b):
            c.out.fill_(3.0)
            c.scores.fill_(0.5)
        torch.cuda.synchronize()
        for c, st in zip((a, b), streams):
            with torch.cuda.stream(st):
                c.run()
        torch.cuda.synchronize()
        for c, (out, scores) in zip((a, b), want):
            assert torch.equal(c.out, out) and torch.equal(c.scores, scores)


@pytest.mark.parametrize("dtype", [BF, F32])
def test_a_captured_step_of_the_cache(dtype):
    """rotation and attention of PagedCache.decode_step, replayed: each token goes to its place, n_ctx counts on."""
    g = torch.Generator().manual_seed(33)
    d = kvr.make_desc(B_, HQ, HKV, 1, 1, dtype)
    turn = _rotation(d, dtype, g)[0]
    caches = []
    k, v = (torch.randn(60, HKV, PAGE, D, generator=g).to(dtype).cuda() for _ in range(2))
    for _ in range(2):
        c = PagedCache(d, n_pages=60, page_size=PAGE, table_cap=ROOM // PAGE, rotation=turn, axes=kvr.make_axes(AXIS))
        c.k.copy_(k)
        c.v.copy_(v)
        c.assign(0, 0, list(range(20)))
        for b in range(1, B_):
            c.begin_with(b, 0, 310, page=19 + b)
        for b in range(B_):
            c.assign(b, 20, list(range(30 + 4 * b, 34 + 4 * b)))
        c.n_ctx.fill_(310)
        c.share([0, B_], [310])
        caches.append(c)
    x = torch.randn(20, B_, HQ + 2 * HKV, D, generator=g).to(dtype).cuda()
    now, pos = x[0].clone(), torch.zeros(3, B_, dtype=torch.int32, device="cuda")
    step = lambda c: c.decode_step(now[:, :HQ], now[:, HQ:HQ + HKV], now[:, HQ + HKV:], pos=pos)
    one, two = caches
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(two)
    for i in range(20):                                          # past the end of a page
        now.copy_(x[i])
        pos.fill_(200 + i)
        step(one)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(one.out, two.out) and torch.equal(one.scores, two.scores)
    assert torch.equal(one.k, two.k) and two.n_ctx.tolist() == [330] * B_


@pytest.mark.parametrize("dtype", [BF, F32])
def test_a_dense_cache_of_copies(dtype):
    """No table: every sequence has a copy of what is shared, of which one is read."""
    g = torch.Generator().manual_seed(34)
    B, n = 7, [2600, 2501, 2500, 2700, 2502, 30, 2503]
    d = kvr.make_desc(B, HQ, HKV, 1, 1, dtype)
    k, v = (torch.randn(B, HKV, 30000, D, generator=g).to(dtype) for _ in range(2))
    for x in (k, v):
        x[1:, :, :2500] = x[0, :, :2500]
    q = torch.randn(B, HQ, D, generator=g).to(dtype)
    pages = kvr.make_pages(d, k.cuda(), v.cuda())
    i32 = lambda x: torch.tensor(x, dtype=torch.int32).cuda()
    grp = kvr.make_groups(i32([0, 7]), i32([2500]))
    out, sc = torch.empty_like(q).cuda(), torch.zeros(B, HKV, 2700, device="cuda")
    ws = torch.empty(max(256, kvr.kvr_attend_shared_workspace_size(d, B, pages, grp, 0, 0, True)), dtype=torch.uint8, device="cuda")
    kvr.kvr_attend_shared(d, q.cuda(), B, None, i32(n), pages, grp, 0, 0, out, sc, 2700, ws)
    ref = R.attend(q, k[:, :, :2701].contiguous(), v[:, :, :2701].contiguous(), None, n, None, d.softmax_scale, 0, 0, 2700, HKV)
    tol = _near(out, ref, dtype)
    assert bool(((sc.cpu().double() - ref["scores"]).abs() <= tol).all())


@pytest.mark.parametrize("dtype", [BF, F32])
def test_a_captured_call_of_many_sequences_follows_lengths_and_groups(dtype):
    """Ends that the join attends to become longer than it takes, and shorter again; groups come and go."""
    g = torch.Generator().manual_seed(35)
    B, Hq, Hkv, pool = 64, 16, 8, 400
    d = kvr.make_desc(B, Hq, Hkv, 1, 1, dtype)
    k, v = (torch.randn(pool, Hkv, PAGE, D, generator=g).to(dtype).cuda() for _ in range(2))
    table = torch.randint(0, pool, (B, 2000), generator=g, dtype=torch.int32)
    table[:, :30] = table[0, :30]                                # 480 tokens
    pages = kvr.make_pages(d, k, v, table.cuda())
    q = torch.randn(B, Hq, D, generator=g).to(dtype).cuda()
    i32 = lambda n: torch.zeros(n, dtype=torch.int32, device="cuda")
    n_ctx, start, common = i32(B), i32(3), i32(2)
    groups = kvr.make_groups(start, common)
    out, scores = torch.empty_like(q), torch.empty(B, Hkv, 1500, device="cuda")
    ws = torch.empty(kvr.kvr_attend_shared_workspace_size(d, B, pages, groups, 0, 0, True), dtype=torch.uint8, device="cuda")
    run = lambda: kvr.kvr_attend_shared(d, q, B, None, n_ctx, pages, groups, 0, 0, out, scores, 1500, ws)
    steps = [([481 + i for i in range(B)], [0, 40, 64], [480, 480]), ([481 + 9 * i for i in range(B)], [0, 64, 64], [480, 0]),
             ([20 * i for i in range(B)], [0, 10, 64], [0, 480]), ([0] * B, [0, 64, 64], [480, 0]), ([1400 - i for i in range(B)], [3, 3, 3], [480, 480]),
             ([481 + i for i in range(B)], [0, 40, 64], [480, 480])]

    def set_to(n, s, c):
        for to, x in ((n_ctx, n), (start, s), (common, c)):
            to.copy_(torch.tensor(x, dtype=torch.int32))
        out.fill_(3.0)
        scores.fill_(0.5)
    set_to(*steps[0])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run()
    want = []
    for s in steps:
        set_to(*s)
        ws.fill_(255)
        run()
        want.append((out.clone(), scores.clone()))
    for s, (o, sc) in zip(steps, want):
        set_to(*s)
        ws.random_(0, 255)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, o) and torch.equal(scores, sc)
        _ = (out.float() @ out.float().transpose(1, 2)).sum().item()
    ref = R.attend(q.cpu(), k.cpu(), v.cpu(), table, steps[2][0], None, d.softmax_scale, 0, 0, 1500, Hkv)
    tol = _near(want[2][0], ref, dtype, torch.full((B, Hkv, 1500), 0.5))
    assert bool(((want[2][1].cpu().double() - 0.5 - ref["scores"]).abs() <= tol).all())

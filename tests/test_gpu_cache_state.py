"""The operators of the uncompressed cache run together, as LayerState and PagedCache run them: a ragged batch of prompts,
decode steps over its pages with a window, and a prompt that is compressed with the scores all its queries left."""
import pytest
import torch

from paper_2512_17917_amd import binding as kvr
from paper_2512_17917_amd.state import LayerState, PagedCache, attend_dense_prompt
from tests import cache_ref as R

pytestmark = [pytest.mark.gpu, pytest.mark.timeout(300)]
D = 128
BF, F32 = torch.bfloat16, torch.float32


def _rotation(d, dtype, g, rot=128, pairs=False):
    inv = 1e6 ** (-torch.arange(rot // 2, dtype=torch.float64) / (rot // 2))
    wq, wk = ((torch.randn(D, generator=g) * 0.2 + 1).to(dtype) for _ in range(2))
    dev = kvr.make_rotation(d, inv.cuda(), q_weight=wq.cuda(), k_weight=wk.cuda(), pairs=pairs)
    return dev, lambda x, w, pos: R.rotate(x, w, pos, inv, 1e-6, pairs), wq, wk


def _near(got, ref, dtype, old=None):
    tol, tol_s = R.attend_bounds(ref, dtype, old)
    err = (got.cpu().double() - ref["out"]).abs()
    assert bool((err <= tol)[ref["rows"]].all()), float((err - tol)[ref["rows"]].max())
    return tol_s


@pytest.mark.parametrize("dtype,window,n_sink", [(BF, 0, 0), (BF, 48, 3), (F32, 0, 0), (F32, 33, 16)])
def test_prompts_then_decode_steps(dtype, window, n_sink):
    """Every stage against float64 of what the stage before it left on the GPU (so that no rounding is counted twice)."""
    g = torch.Generator().manual_seed(5)
    B, Hq, Hkv, ps, cap = 3, 8, 2, 16, 12
    d = kvr.make_desc(B, Hq, Hkv, 1, 1, dtype)
    turn, plain, wq, wk = _rotation(d, dtype, g)
    c = PagedCache(d, n_pages=B * cap + 2, page_size=ps, table_cap=cap, rotation=turn, window=window, n_sink=n_sink)
    order = torch.randperm(B * cap + 2, generator=g)[:B * cap].view(B, cap).tolist()
    for b in range(B):
        c.assign(b, 0, order[b])
    lens = [150, 1, 77]
    q_start = [0]
    for n in lens:
        q_start.append(q_start[-1] + n)
    fused = torch.randn(q_start[-1], Hq + 2 * Hkv, D, generator=g).to(dtype)
    c.n_ctx += torch.tensor(lens, dtype=torch.int32).cuda()
    qs = torch.tensor(q_start, dtype=torch.int32).cuda()
    f = fused.cuda()
    out = c.prompt(f[:, :Hq], f[:, Hq:Hq + Hkv], f[:, Hq + Hkv:], qs)
    pos = torch.cat([torch.arange(n) for n in lens])
    ref_k, size = plain(fused[:, Hq:Hq + Hkv], wk, pos)
    table, kp, vp = c.table.cpu(), c.k.cpu(), c.v.cpu()
    for b in range(B):
        for t in range(lens[b]):
            page, row = R.token_row(kp, table, b, t)
            i = q_start[b] + t
            assert bool(((kp[page, :, row].double() - ref_k[i]).abs() <= R.rotate_bound(ref_k[i], size[i], dtype)).all())
            assert torch.equal(vp[page, :, row], fused[i, Hq + Hkv:])
    turned = torch.empty(q_start[-1], Hq, D, dtype=dtype).cuda()
    kvr.kvr_rotate(d, turn, f[:, :Hq], None, None, q_start[-1], qs, c.n_ctx, turned)
    ref = R.attend(turned.cpu(), kp, vp, table, lens, q_start, d.softmax_scale, window, n_sink, c.n_cap, Hkv)
    tol_s = _near(out, ref, dtype)
    assert bool(((c.scores.cpu().double() - ref["scores"]).abs() <= tol_s).all())
    for step in range(20):                                       # across the ends of pages, and of the window
        before = c.scores.cpu()
        x = torch.randn(B, Hq + 2 * Hkv, D, generator=g).to(dtype).cuda()
        out = c.decode_step(x[:, :Hq], x[:, Hq:Hq + Hkv], x[:, Hq + Hkv:])
        lens = [n + 1 for n in lens]
        kp, vp = c.k.cpu(), c.v.cpu()
        for b in range(B):
            page, row = R.token_row(kp, table, b, lens[b] - 1)
            assert torch.equal(vp[page, :, row], x[b, Hq + Hkv:].cpu())
        ref = R.attend(c.q.cpu(), kp, vp, table, lens, None, d.softmax_scale, window, n_sink, c.n_cap, Hkv)
        tol_s = _near(out, ref, dtype, before)
        assert bool(((c.scores.cpu().double() - before.double() - ref["scores"]).abs() <= tol_s).all())
    assert c.n_ctx.tolist() == lens


@pytest.mark.parametrize("dtype", [BF, F32])
def test_prompt_compressed_with_its_own_scores(dtype):
    """from_prefill with the prompt's queries: the outputs and scores of causal attention; the tokens that leave are those
    with the lowest scores; where none leaves, a decode step with a rotation attends over all of them."""
    g = torch.Generator().manual_seed(9)
    B, Hq, Hkv, N = 2, 8, 2, 130
    d = kvr.make_desc(B, Hq, Hkv, 3, 16, dtype, seed=3)
    turn, plain, wq, wk = _rotation(d, dtype, g)
    K, V = (torch.randn(B, Hkv, N, D, generator=g).to(dtype) for _ in range(2))
    q = torch.randn(B, N, Hq, D, generator=g).to(dtype)
    ref = R.attend(q.flatten(0, 1), K, V, None, [N] * B, [0, N, 2 * N], d.softmax_scale, 0, 0, N, Hkv)
    for recent, cand in ((40, 30), (N, 10)):
        ls, info = LayerState.from_prefill(d, K.cuda(), V.cuda(), None, n_recent=recent, k_candidate=cand, max_new_tokens=4,
                                           q_prompt=q.cuda())
        tol_s = _near(info["out"].flatten(0, 1), ref, dtype)
        sc = ls.scores.cpu()
        assert bool(((sc[:, :, :N].double() - ref["scores"]).abs() <= tol_s).all())
        gone = max(N - recent - cand, 0)
        assert bool((ls.n_vague.cpu() == gone).all())
        for b in range(B):
            for h in range(Hkv):
                mine = sc[b, h, :N - recent] if gone else sc[b, h, :0]
                stays = set(torch.topk(mine, cand).indices.tolist()) if gone else set()
                assert set(ls.vague_pos[b, h, :gone].tolist()) == set(range(N - recent)) - stays if gone else True
    # the second state kept every token: one step with the projections of a new one
    x = torch.randn(B, Hq + 2 * Hkv, D, generator=g).to(dtype)
    xd = x.cuda()
    v_new = xd[:, Hq + Hkv:].contiguous()
    out = ls.decode_step(xd[:, Hq:Hq + Hkv], v_new, xd[:, :Hq], rotation=turn)
    q_ref, q_size = plain(x[:, :Hq], wq, torch.full((B,), N))
    k_ref, k_size = plain(x[:, Hq:Hq + Hkv], wk, torch.full((B,), N))
    qt, kt = ls.q_turned.cpu(), ls.k_turned.cpu()
    assert bool(((qt.double() - q_ref).abs() <= R.rotate_bound(q_ref, q_size, dtype)).all())
    assert bool(((kt.double() - k_ref).abs() <= R.rotate_bound(k_ref, k_size, dtype)).all())
    K1, V1 = torch.cat([K, kt[:, :, None]], 2), torch.cat([V, x[:, Hq + Hkv:, None]], 2)
    one = R.attend(qt, K1, V1, None, [N + 1] * B, None, d.softmax_scale, 0, 0, N + 4, Hkv)
    _near(out, one, dtype)


def test_pages_to_a_compressed_state():
    """PagedCache.dense and its scores are what from_prefill takes: the same state as from the dense cache itself."""
    g = torch.Generator().manual_seed(13)
    B, Hq, Hkv, ps, N = 2, 8, 2, 24, 100
    d = kvr.make_desc(B, Hq, Hkv, 3, 8, BF, seed=1)
    c = PagedCache(d, n_pages=12, page_size=ps, table_cap=6)
    for b in range(B):
        c.assign(b, 0, [b + 2 * i for i in range(6)])
    q, k, v = (torch.randn(B * N, h, D, generator=g).to(BF).cuda() for h in (Hq, Hkv, Hkv))
    qs = torch.tensor([0, N, 2 * N], dtype=torch.int32).cuda()
    c.n_ctx += N
    out = c.prompt(q, k, v, qs)
    K, V = c.dense(N)
    assert torch.equal(K, k.view(B, N, Hkv, D).transpose(1, 2)) and torch.equal(V, v.view(B, N, Hkv, D).transpose(1, 2))
    scores = torch.zeros(B, Hkv, N).cuda()
    same = attend_dense_prompt(d, q.view(B, N, Hq, D), K, V, c.n_ctx, scores)
    ref = R.attend(q.cpu(), K.cpu(), V.cpu(), None, [N] * B, [0, N, 2 * N], d.softmax_scale, 0, 0, N, Hkv)
    _near(same.flatten(0, 1), ref, BF)
    _near(out, ref, BF)
    tol_s = R.attend_bounds(ref, BF)[1]
    assert bool(((c.scores[:, :, :N].cpu().double() - ref["scores"]).abs() <= tol_s).all())
    a, _ = LayerState.from_prefill(d, K, V, None, n_recent=20, k_candidate=20, max_new_tokens=2, init_scores=c.scores[:, :, :N])
    assert bool((a.n_vague == N - 40).all())
    kept = a.ret_pos[:, :, :40].cpu()
    for b in range(B):
        for h in range(Hkv):
            assert torch.equal(a.k_ret[b, h, :40].cpu(), K[b, h].cpu()[kept[b, h].long()])

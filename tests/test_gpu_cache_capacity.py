"""The largest sizes that the operators of the uncompressed cache accept are launched whole."""
import pytest
import torch

from paper_2512_17917_amd import binding as kvr
from tests import cache_ref as R
from tests.test_gpu_cache_ops import _attend, _dev, _normal, _starts

pytestmark = [pytest.mark.gpu, pytest.mark.timeout(300)]
D = 128
BF, F32 = torch.bfloat16, torch.float32


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

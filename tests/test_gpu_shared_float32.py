"""kvr_attend_shared in float32, one head a key head: logits whose products, added one after another, would lose their lower bits."""
import pytest
import torch

from paper_2512_17917_amd import binding as kvr
from tests.test_gpu_shared import D, F32, ROOM, Batch, one

pytestmark = [pytest.mark.gpu, pytest.mark.timeout(300)]

CASES = [  # groups, heads, page, room: by the kernels for small caches and those that share
    ([(640, one(1641, 2100, 900))], (8, 8), 16, 0),
    ([(640, one(1641, 2100, 900))], (8, 8), 24, 0),
    ([(640, one(1641, 2100, 900))], (8, 8), 16, ROOM),
    ([(640, one(1641, 2100, 900))], (8, 2), 24, ROOM),
]


@pytest.mark.parametrize("case", range(len(CASES)))
def test_a_large_product_beside_small_ones(case):
    """Keys (2^24, 0, ...) at even tokens, with 127 times 0.2 behind it at odd ones, values 1 and -1: odd tokens' logits are 25.4 2^-8
    = 0.0992 above the others', and the output about -tanh(0.0496) = -0.0496.  Four of the small products and fewer are lost beside 2^24,
    where floats are 2 apart: all of them in one sum.  In four sums 31 of them are, 6.2, and two last additions are off by 1 each; the
    logits in powers of two, near 94548, by half of 2^-7 each.  Of the odd tokens' logit (8.2 + 0.0054 2^8) 2^-8 = 0.0375, of the output
    half as much at most; 1e-5 for the rest."""
    groups, heads, page, room = CASES[case]
    b = Batch(groups, heads, page, F32, 190 + case, rows=False, room=room)
    b.q.fill_(1.0)
    b.k.zero_()
    for s, n in enumerate(b.n):
        for j in range(n):
            at, row = b.table[s, j // page], j % page
            b.k[at, :, row, 1:] = 0.2 * (j % 2)
            b.k[at, :, row, 0] = 2.0 ** 24
            b.v[at, :, row] = 1 - 2 * (j % 2)
    d = kvr.make_desc(b.B, b.Hq, b.Hkv, 1, 1, F32, softmax_scale=2.0 ** -8)
    i32 = lambda x: torch.tensor(x, dtype=torch.int32).cuda()
    pages, groups = kvr.make_pages(d, b.k.cuda(), b.v.cuda(), b.table.cuda()), kvr.make_groups(i32(b.start), i32(b.common))
    out = torch.zeros(b.rows, b.Hq, D).cuda()
    ws = torch.empty(max(256, kvr.kvr_attend_shared_workspace_size(d, b.rows, pages, groups, 0, 0, False)), dtype=torch.uint8).cuda()
    kvr.kvr_attend_shared(d, b.q.cuda(), b.rows, None, i32(b.n), pages, groups, 0, 0, out, None, 0, ws)
    for s, n in enumerate(b.n):
        few, many = (n + 1) // 2, n // 2                         # even tokens, odd ones
        w = torch.tensor(127 * 0.2 * 2.0 ** -8, dtype=torch.float64).exp() * many
        ref = (few - w) / (few + w)
        err = (out[s].cpu().double() - ref).abs().max()
        assert float(err) <= 0.0188 + 1e-5, (s, float(err))

"""kvr_attend_shared in bf16 keeps a weight's lower bits where a sequence has one new row: its error is that of float32 sums, not half a
step of bf16 a weight.  (Of several rows it rounds weights as kvr_attend_prompt does.)"""
import math

import pytest
import torch

from paper_2512_17917_amd import binding as kvr
from tests import cache_ref as R
from tests.test_gpu_shared import BF, D, Batch, one

pytestmark = [pytest.mark.gpu, pytest.mark.timeout(300)]

CASES = [  # groups, heads, page, by q_start: few columns and many, of a group and of a sequence, pages of whole eights and others
    ([(640, one(*[641 + 70 * i for i in range(6)]))], (8, 2), 16, False),
    ([(640, one(*[641 + 70 * i for i in range(6)]))], (8, 2), 7, False),
    ([(640, one(*[641 + 70 * i for i in range(20)]))], (16, 2), 64, False),
    ([(640, [(700 + i, 1 + i % 5) for i in range(9)])], (8, 2), 16, True),
    ([(640, [(700 + 50 * i, 1 + i % 8) for i in range(9)])], (16, 2), 5, True),
    ([(0, one(900, 70, 333))], (4, 2), 8, False),
]


def _flat(case, delta):
    """Logits 0 at even tokens and -delta at odd ones (channel 0 alone), values 1 and -1: nearly all of the sum cancels, and what
    rounds one token's weight rounds every other's the same way."""
    groups, heads, page, rows = CASES[case]
    b = Batch(groups, heads, page, BF, 130 + case, rows=rows)
    b.q.zero_()
    b.q[:, :, 0] = 1
    b.k.zero_()
    for s, n in enumerate(b.n):
        for j in range(n):
            at, row = R.token_row(b.k, b.table, s, j)
            b.k[at, :, row, 0] = -delta * (j % 2)
            b.v[at, :, row] = 1 - 2 * (j % 2)
    return b


def _attend(b):
    d = kvr.make_desc(b.B, b.Hq, b.Hkv, 1, 1, BF, softmax_scale=1.0)
    i32 = lambda x: torch.tensor(x, dtype=torch.int32).cuda()
    pages = kvr.make_pages(d, b.k.cuda(), b.v.cuda(), b.table.cuda())
    groups = kvr.make_groups(i32(b.start), i32(b.common))
    out = torch.zeros(b.rows, b.Hq, D, dtype=BF).cuda()
    ws = torch.randint(0, 256, (kvr.kvr_attend_shared_workspace_size(d, b.rows, pages, groups, 0, 0, False),), dtype=torch.uint8).cuda()
    kvr.kvr_attend_shared(d, b.q.cuda(), b.rows, None if b.q_start is None else i32(b.q_start), i32(b.n), pages, groups, 0, 0, out, None, 0, ws)
    return out.cpu().double(), R.attend(b.q, b.k, b.v, b.table, b.n, b.q_start, 1.0, 0, 0, 0, b.Hkv)


@pytest.mark.parametrize("delta", [3 / 512, 5 / 512])
@pytest.mark.parametrize("case", range(len(CASES)))
def test_weights_that_bf16_rounds_one_way(case, delta):
    """exp(-3/512) = 0.99416 and exp(-5/512) = 0.99028 lie 0.0019 from bf16's next (steps of 2^-8): sums off by a thousandth, were
    the weights rounded to it.  The bound: half a step of the output, the float32 bounds of attend_bounds, and 2^-15 a weight (two
    parts in bf16, the upper one cut off, the lower one, below 2^-7 of it, rounded).  Of several rows: half a step a weight."""
    out, ref = _attend(_flat(case, delta))
    err = (out - ref["out"]).abs()
    if CASES[case][3]:
        assert bool((err <= R.attend_bounds(ref, BF)[0]).all())
        return
    rel = 2 * (ref["e"] + 2.0 ** -16) + 2.0 ** -14 + 2.0 ** -15
    tol = R.half_step(BF) * ref["out"].abs() + rel * 1.01 * ref["weight"]
    assert float(tol.max()) < 3e-4                               # (a thousandth would be seen)
    assert bool((err <= tol).all()), float((err - tol).max())


@pytest.mark.parametrize("what", [math.inf, -math.inf])
@pytest.mark.parametrize("case", range(len(CASES)))
def test_an_infinite_value_that_all_see_is_every_columns(case, what):
    """Of weights with no lower bits (all are 1): 0 times infinity is added nowhere."""
    b = _flat(case, 0.0)
    at, row = R.token_row(b.v, b.table, 0, 40)
    b.v[at, :, row, 9] = what
    out, ref = _attend(b)
    inf = torch.isinf(ref["out"])
    assert bool(inf.any()) and torch.equal(out[inf], ref["out"][inf]) and torch.equal(torch.isfinite(out), ~inf)

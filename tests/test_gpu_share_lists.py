"""A step of PagedCache captured while groups were given by lists: it follows the lists given later, and shares nothing once there are none."""
import pytest
import torch

from paper_2512_17917_amd import binding as kvr
from paper_2512_17917_amd.state import PagedCache
from tests import cache_ref as R
from tests.test_gpu_cache_state import _near
from tests.test_gpu_shared import ROOM

pytestmark = [pytest.mark.gpu, pytest.mark.timeout(300)]
D, B, HQ, HKV, PAGE = 128, 6, 8, 2, 16
BF, F32 = torch.bfloat16, torch.float32


@pytest.mark.parametrize("dtype", [BF, F32])
def test_a_captured_step_follows_the_lists(dtype):
    g = torch.Generator().manual_seed(41)
    d = kvr.make_desc(B, HQ, HKV, 1, 1, dtype)
    c = PagedCache(d, n_pages=100, page_size=PAGE, table_cap=ROOM // PAGE)
    for pool in (c.k, c.v):
        pool.copy_(torch.randn(100, HKV, PAGE, D, generator=g).to(dtype))

    def begin(of):                                               # sequence b's first 320 tokens are those of document of[b]
        for b in range(B):
            c.assign(b, 0, list(range(20 * of[b], 20 * of[b] + 20)))
            c.assign(b, 20, [60 + b])
        c.n_ctx.fill_(321)
    step = lambda: c.decode_step(*x)
    x = [torch.randn(B, heads, D, generator=g).to(dtype).cuda() for heads in (HQ, HKV, HKV)]
    begin([0, 0, 0, 1, 1, 1])
    c.share([0, 3, 6], [320, 320])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for of, lists in (([0, 0, 0, 1, 1, 1], ([0, 3, 6], [320, 320])), ([0, 0, 1, 1, 1, 1], ([0, 2, 6], [320, 320])),
                      ([2, 0, 1, 1, 1, 0], ([2, 5], [320])), ([0, 1, 2, 0, 1, 2], (None, None)), ([2] * 6, ([0, 6], [320])),
                      ([0, 1, 2, 1, 2, 0], (torch.tensor([3, 3], dtype=torch.int32).cuda(), torch.tensor([9], dtype=torch.int32).cuda()))):
        begin(of)
        c.share(*lists)
        for t in x:
            t.copy_(torch.randn(t.shape, generator=g))
        trash = [torch.randint(0, 6, (7,), dtype=torch.int32).cuda() for _ in range(50)]      # where freed lists might have been
        before = c.scores.cpu()
        graph.replay()
        torch.cuda.synchronize()
        assert c.n_ctx.tolist() == [322] * B
        ref = R.attend(x[0].cpu(), c.k.cpu(), c.v.cpu(), c.table.cpu(), [322] * B, None, d.softmax_scale, 0, 0, 400, HKV)
        tol = _near(c.out, ref, dtype, before[:, :, :400])
        assert bool(((c.scores[:, :, :400].cpu().double() - before[:, :, :400].double() - ref["scores"]).abs() <= tol).all()), of
        del trash

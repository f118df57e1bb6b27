"""One captured call of the cache's operators, replayed over sequences whose lengths have changed since, and calls on two streams at
once: the lengths are the device's affair, and nothing is shared but what the caller shares."""
import pytest
import torch

from paper_2512_17917_amd import binding as kvr
from tests.test_gpu_cache_ops import _normal

pytestmark = [pytest.mark.gpu, pytest.mark.timeout(300)]
D = 128
BF, F32 = torch.bfloat16, torch.float32
ROOM, PAGE, B, HQ, HKV, ROWS = 8192, 16, 3, 8, 2, 640
LENGTHS = [([500, 30, 0], [500, 30, 0]), ([700, 31, 8192], [200, 1, 3]), ([1, 0, 2], [1, 0, 2]), ([8192, 5000, 900], [640, 0, 0]),
           ([0, 0, 0], [0, 0, 0]), ([500, 30, 0], [500, 30, 0])]


class _Call:
    def __init__(self, which, dtype, window, sink, seed):
        g = torch.Generator().manual_seed(seed)
        self.which, self.window, self.sink = which, window, sink
        self.d = kvr.make_desc(B, HQ, HKV, 1, 1, dtype)
        each = ROOM // PAGE
        self.k, self.v = (_normal(g, B * each, HKV, PAGE, D, dtype=dtype).cuda() for _ in range(2))
        self.table = torch.randperm(B * each, generator=g).to(torch.int32).view(B, each).cuda()
        self.pages = kvr.make_pages(self.d, self.k, self.v, self.table)
        self.rows = ROWS if which == "prompt" else B
        self.q = _normal(g, self.rows, HQ, D, dtype=dtype).cuda()
        self.out = torch.empty_like(self.q)
        self.scores = torch.empty(B, HKV, ROOM, device="cuda")
        self.n_ctx = torch.zeros(B, dtype=torch.int32, device="cuda")
        self.q_start = torch.zeros(B + 1, dtype=torch.int32, device="cuda")
        if which == "prompt":
            n = kvr.kvr_attend_prompt_workspace_size(self.d, self.rows, self.pages, window, sink, True)
        else:
            n = kvr.kvr_attend_paged_workspace_size(self.d, self.pages, window, sink, True)
        self.ws = torch.empty(max(n, 256), dtype=torch.uint8, device="cuda")

    def set(self, n, new):
        self.n_ctx.copy_(torch.tensor(n, dtype=torch.int32))
        starts = [0]
        for y in new:
            starts.append(starts[-1] + y)
        self.q_start.copy_(torch.tensor(starts, dtype=torch.int32))
        self.out.fill_(3.0)
        self.scores.fill_(0.5)

    def run(self):
        if self.which == "prompt":
            kvr.kvr_attend_prompt(self.d, self.q, self.rows, self.q_start, self.n_ctx, self.pages, self.window, self.sink, self.out,
                                  self.scores, ROOM, self.ws)
        else:
            kvr.kvr_attend_paged(self.d, self.q, self.n_ctx, self.pages, self.window, self.sink, self.out, self.scores, ROOM, self.ws)

    def results(self):
        return self.out.clone(), self.scores.clone()


@pytest.mark.parametrize("window,sink", [(0, 0), (300, 20)])
@pytest.mark.parametrize("which,dtype", [("prompt", BF), ("prompt", F32), ("paged", BF), ("paged", F32)])
def test_a_captured_call_follows_the_lengths(which, dtype, window, sink):
    c = _Call(which, dtype, window, sink, 5)
    want = []
    for n, new in LENGTHS:
        c.set(n, new)
        c.ws.fill_(255)
        c.run()
        want.append(c.results())
    assert torch.equal(want[0][0], want[-1][0]) and torch.equal(want[0][1], want[-1][1])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        c.run()
    for (n, new), (out, scores) in zip(LENGTHS, want):
        c.set(n, new)
        c.ws.random_(0, 255)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(c.out, out) and torch.equal(c.scores, scores), (n, new)
        _ = (c.out.float() @ c.out.float().transpose(1, 2)).sum().item()


def test_calls_on_two_streams_at_once():
    """Each with a workspace and results of its own, over the same cache."""
    a, b = _Call("prompt", BF, 0, 0, 6), _Call("prompt", BF, 300, 20, 6)
    b.k, b.v, b.table, b.pages = a.k, a.v, a.table, a.pages
    for c, (n, new) in ((a, LENGTHS[1]), (b, LENGTHS[3])):
        c.set(n, new)
        c.run()
    want = [c.results() for c in (a, b)]
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for _ in range(5):
        for c, (n, new) in ((a, LENGTHS[1]), (b, LENGTHS[3])):
            c.set(n, new)
        torch.cuda.synchronize()
        for _ in range(3):
            for c, s in zip((a, b), streams):
                with torch.cuda.stream(s):
                    c.out.fill_(3.0)
                    c.scores.fill_(0.5)
                    c.run()
        torch.cuda.synchronize()
        for c, (out, scores) in zip((a, b), want):
            assert torch.equal(c.out, out) and torch.equal(c.scores, scores)

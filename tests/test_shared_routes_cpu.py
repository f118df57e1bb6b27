"""That the GPU tests written for the kernels of kvr_attend_shared reach them: the call goes by sizes, and small caches take other
kernels."""
import subprocess

import pytest

from paper_2512_17917_amd import build as B
from tests import launches
from tests.test_gpu_shared import BF, F32, Batch
from tests import test_gpu_shared_weights as weights
from tests.test_shared_cpu import PROBE


@pytest.fixture(scope="module")
def ask(tmp_path_factory):
    return launches.build_probe(tmp_path_factory.mktemp("launches"))


def _names(ask, calls, *want):
    for call, kernels in zip(calls, ask(calls)):
        scores = kernels[2:] if call["scores"] else []          # (of several rows a sequence one launch or two)
        assert len(kernels) - len(scores) == 2 and bool(scores) == bool(call["scores"]), (call, kernels)
        assert all(w in k for w, k in zip(want, kernels)), (call, kernels)


def test_weights(ask):
    for groups, heads, page, rows in weights.CASES:
        b = Batch(groups, heads, page, BF, 0, rows=rows)
        _names(ask, [launches.call_of(b, False, scores=False)], "shared_bf16_kernel", "shared_join_kernel")


@pytest.mark.parametrize("f32", [0, 1])
def test_steps_captured_with_lists(ask, f32):
    from tests import test_gpu_share_lists as t
    call = dict(f32=f32, B=t.B, Hq=t.HQ, Hkv=t.HKV, rows=t.B, by_start=0, page=t.PAGE, cols=t.ROOM // t.PAGE, window=0, sink=0, groups=t.B, scores=1)
    _names(ask, [call], "shared_f32_kernel" if f32 else "shared_bf16_kernel", "shared_join_kernel", "shared_scores_kernel")


@pytest.mark.parametrize("f32", [0, 1])
def test_windows(ask, f32):
    from tests import test_gpu_shared_windows as t
    attend, dtype = ("shared_f32_kernel", F32) if f32 else ("shared_bf16_kernel", BF)
    for case in range(len(t.WINDOWS)):
        b, window, sink = t.batch(case, dtype)
        calls = [launches.call_of(b, f32, window, sink, scores) for scores in (True, False)]
        by_rows = b.q_start is not None
        join = "shared_join_kernel" if by_rows else "shared_own_kernel"
        _names(ask, calls[:1], attend, join, *(["scores"] if by_rows else ["shared_scores_kernel"]))
        _names(ask, calls[1:], attend, join)
    call = dict(f32=f32, B=t.B_, Hq=t.HQ, Hkv=t.HKV, rows=t.ROWS, by_start=1, page=t.PAGE, cols=t.TOKENS // t.PAGE, window=t.WINDOW, sink=t.SINK,
                groups=3, scores=1)
    _names(ask, [call], attend, "shared_join_kernel", "scores")
    _names(ask, [dict(call, rows=t.B_, by_start=0)], attend, "", "shared_scores_kernel")


def test_lists_that_are_filled_again(ask):
    from tests import test_gpu_shared_refill as t
    for case in range(len(t.CASES)):
        s = t.Setup(case)
        for dtype in t.CASES[case][1]:
            call = dict(f32=dtype == F32, B=s.B, Hq=s.heads[0], Hkv=s.heads[1], rows=s.rows, by_start=s.most > 0, page=s.page, cols=s.cols, window=0,
                        sink=0, groups=s.groups, scores=1)
            _names(ask, [call], "shared_f32_kernel" if dtype == F32 else "shared_bf16_kernel", "shared_", "scores")


def test_lists_that_are_filled_again_are_full(tmp_path):
    """More pieces, or tiles with those of queries, in some workgroup than its lists hold, and cuts between queries and tokens."""
    from tests import test_gpu_shared_refill as t
    src, exe = str(tmp_path / "probe.hip"), str(tmp_path / "probe")
    open(src, "w").write(PROBE)
    subprocess.run([B._hipcc(), "--offload-host-only", "-std=c++17", "-I", B.CSRC, src, "-o", exe], check=True, capture_output=True)
    cuts = 0
    for case, (name, dtypes, _, page, *_) in enumerate(t.CASES):
        s = t.Setup(case)
        Hq, Hkv = s.heads
        starts = [0]
        for y in s.y:
            starts.append(starts[-1] + y)
        for which, wgs, cols in ((0, 256, 256), (1, 512, 16), (2, 512, 64)):
            if (which == 1 and F32 not in dtypes) or (which == 2 and s.most):
                continue
            words = [which, wgs, s.B, Hq // Hkv, Hkv, s.rows, s.cols * page, 0, 0, s.groups, 0 if s.most or s.B * Hkv < 512 else 256, *s.n, int(s.most > 0),
                     *(starts if s.most else []), *s.start, *s.common]
            lines = subprocess.run([exe], input=" ".join(map(str, words)) + "\n", capture_output=True, text=True, check=True).stdout.splitlines()
            pieces, tiles = {}, {}
            for line in lines[1:-1]:
                w, _, _, _, _, _, some, _, _, _, _, _, _, _, i0, i1, _ = map(int, line.split())
                pieces[w] = pieces.get(w, 0) + 1
                if i0 < i1:
                    queries = 0 if some <= 16 else 1 if some <= 128 else 2
                    first = sum(tiles.setdefault(w, []))
                    at = (128 if page % 8 == 0 else 24) - first
                    cuts += which == 0 and pieces[w] <= 64 and 0 < at <= queries
                    tiles[w].append(queries + i1 - i0)
            if "pieces" in name:
                assert max(pieces.values()) > 64, (name, which)
            elif which == 0:
                assert max(map(sum, tiles.values())) > (128 if page % 8 == 0 else 24), name
    assert cuts > 20


def test_launches_stay_within_their_lds_limit(ask):
    """More than 64 KB only where the limit was raised for the kernel, on the device of the call."""
    call = dict(B=64, Hq=32, Hkv=8, rows=64, page=16, cols=1000, window=0, sink=0, groups=1)
    calls = [dict(call, f32=f32, page=page, scores=scores, by_start=by_start, device=dev)
             for dev in (0, 3, 0) for page in (16, 7) for f32 in (0, 1) for scores in (0, 1) for by_start in (0, 1)]
    for c, kernels, lds in zip(calls, ask(calls), ask.lds):
        assert "shared" in kernels[0] and all(asked <= most <= 160 * 1024 for asked, most in lds), (c, kernels, lds)
        assert c["f32"] or lds[0][0] > 65536


def test_float32(ask):
    from tests import test_gpu_shared_float32 as t
    for groups, heads, page, room in t.CASES:
        b = Batch(groups, heads, page, F32, 0, rows=False, room=room)
        _names(ask, [launches.call_of(b, True, scores=False)], "shared_f32_kernel" if room else "12paged_kernel", "join_kernel")

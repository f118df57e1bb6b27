"""That the GPU tests written for the kernels of kvr_attend_shared reach them: the call goes by sizes, and small caches take other
kernels."""
import pytest

from tests import launches
from tests.test_gpu_shared import BF, Batch
from tests import test_gpu_shared_weights as weights


@pytest.fixture(scope="module")
def ask(tmp_path_factory):
    return launches.build_probe(tmp_path_factory.mktemp("launches"))


def _names(ask, calls, *want):
    for call, kernels in zip(calls, ask(calls)):
        assert len(kernels) == len(want) and all(w in k for w, k in zip(want, kernels)), (call, kernels)


def test_weights(ask):
    for groups, heads, page, rows in weights.CASES:
        b = Batch(groups, heads, page, BF, 0, rows=rows)
        _names(ask, [launches.call_of(b, False, scores=False)], "shared_bf16_kernel", "shared_join_kernel")


@pytest.mark.parametrize("f32", [0, 1])
def test_steps_captured_with_lists(ask, f32):
    from tests import test_gpu_share_lists as t
    call = dict(f32=f32, B=t.B, Hq=t.HQ, Hkv=t.HKV, rows=t.B, by_start=0, page=t.PAGE, cols=t.ROOM // t.PAGE, window=0, sink=0, groups=t.B, scores=1)
    _names(ask, [call], "shared_f32_kernel" if f32 else "shared_bf16_kernel", "shared_join_kernel", "shared_scores_kernel")

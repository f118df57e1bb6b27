"""What the binding and the cache's classes refuse, on the CPU: calls that would read past an operand, mix up tokens or drop scores."""
import pytest
import torch

from paper_2512_17917_amd import binding as kvr
from tests.test_cache_fast_cpu import Fake, _desc, _rotate_args, fast        # noqa: F401


@pytest.mark.parametrize("route", ["c", "python"])
@pytest.mark.parametrize("which", ["q_weight", "k_weight"])
def test_a_rotation_whose_weights_are_of_another_type_is_refused(fast, monkeypatch, route, which):       # noqa: F811
    """128 weights in bf16, 256 bytes, are not 512 bytes of float32."""
    _, got = fast
    if route == "python":
        monkeypatch.setattr(kvr, "_fast", None)
    d = _desc()
    wide = kvr.make_desc(3, 8, 2, 1, 1, torch.float32, hash_params=[(1, 2, 3, 4)])
    inv = Fake(torch.float64, (64,), 0xc000)
    for made, used in ((d, wide), (wide, d)):
        rot = kvr.make_rotation(made, inv, **{which: Fake(kvr._torch_dtype(made), (128,), 0xd000)})
        a = _rotate_args(v=None)
        for name in ("q", "k", "q_out", "k_out"):
            a[name] = Fake(kvr._torch_dtype(used), a[name].shape, a[name].data_ptr(), a[name].stride())
            a[name]._c = True
        with pytest.raises(ValueError):
            kvr.kvr_rotate(used, rot, *a.values())
        assert not got
        # frequencies alone are the same for both
        kvr.kvr_rotate(used, kvr.make_rotation(made, inv), *a.values())
        assert len(got) == 1
        got.clear()

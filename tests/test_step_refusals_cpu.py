"""Decode steps that are refused, on the CPU: the token is not counted, so that the same step with right arguments follows."""
import pytest
import torch

from paper_2512_17917_amd import binding as kvr
from paper_2512_17917_amd.state import LayerState, PagedCache

AXES = kvr.make_axes([0] * 64)
POS = torch.zeros(1, 2, dtype=torch.int32)


def _paged(axes=None):
    c = PagedCache.__new__(PagedCache)
    c.desc = kvr.make_desc(2, 8, 2, 3, 5, torch.bfloat16, seed=1)
    c.rotation, c.n_ctx, c.q, c.pages, c.groups, c.axes = kvr.make_rotation(c.desc), torch.full((2,), 7, dtype=torch.int32), None, None, None, axes
    return c


def _layer():
    s = LayerState.__new__(LayerState)
    s.desc = kvr.make_desc(2, 8, 2, 3, 5, torch.bfloat16, seed=1)
    s.device, s.dtype = torch.device("cpu"), torch.bfloat16
    s.k_turned, s.q_turned, s.n_ctx, s.r_size = None, None, torch.full((2,), 7, dtype=torch.int32), 3
    return s


TOKENS = torch.zeros(2, 2, 128, dtype=torch.bfloat16), torch.zeros(2, 2, 128, dtype=torch.bfloat16), torch.zeros(2, 8, 128, dtype=torch.bfloat16)


@pytest.mark.parametrize("axes,pos", [(AXES, None), (None, POS), (AXES, POS), (None, None)])
@pytest.mark.parametrize("bump", [True, False])
def test_a_refused_step_of_the_cache_counts_no_token(axes, pos, bump):
    """Half a pair, and (both or none) tensors that are not on the GPU."""
    c = _paged(axes)
    k, v, q = TOKENS
    with pytest.raises(Exception):
        c.decode_step(q, k, v, bump_n_ctx=bump, pos=pos)
    assert c.n_ctx.tolist() == [7, 7]


@pytest.mark.parametrize("axes,pos", [(AXES, None), (None, POS), (AXES, POS), (None, None)])
@pytest.mark.parametrize("bump", [True, False])
def test_a_refused_step_of_a_layer_counts_no_token(axes, pos, bump):
    s = _layer()
    with pytest.raises(Exception):
        s.decode_step(*TOKENS, bump_n_ctx=bump, rotation=kvr.make_rotation(s.desc), axes=axes, pos=pos)
    assert s.n_ctx.tolist() == [7, 7] and s.r_size == 3


@pytest.mark.parametrize("axes,pos", [(AXES, None), (None, POS), (AXES, POS)])
def test_axes_and_positions_without_a_rotation_are_refused(axes, pos):
    """(They would be dropped, and the token attended to as it comes.)"""
    s = _layer()
    s.step_update = s.append = s.attend = lambda *a, **kw: None
    s.n_recent, s.slack, s.ret_cap, s.evict_cap = 4, 0, 10, 8
    with pytest.raises(ValueError):
        s.decode_step(*TOKENS, axes=axes, pos=pos)
    assert s.n_ctx.tolist() == [7, 7] and s.r_size == 3
    s.decode_step(*TOKENS)
    assert s.n_ctx.tolist() == [8, 8]


def test_a_refused_rotation_leaves_buffers_of_the_right_size():
    """(Too small ones, made after the operands of a call that is refused, would refuse every later call.)"""
    s = _layer()
    k, v, q = TOKENS
    with pytest.raises(Exception):
        s.rotate(k[:1], q[:, :3], kvr.make_rotation(s.desc))
    for buffer, like in ((s.k_turned, k), (s.q_turned, q)):
        assert buffer is None or buffer.shape == like.shape


@pytest.mark.parametrize("bump", [True, False])
@pytest.mark.parametrize("fused", [True, False, None])
def test_a_token_that_is_refused_is_not_in_the_recent_queue(bump, fused):
    """A key or value that the update refuses: neither n_ctx nor the queue's size has moved, and the step can be made again."""
    s = _layer()
    s.n_recent, s.slack, s.ret_cap, s.evict_cap, done = 4, 0, 10, 8, []
    s.select = s.encode = s.attend = lambda *a, **kw: done.append(1)
    refuse = True

    def update(k, v):
        if refuse:
            raise ValueError("k_new")
    s.step_update = s.append = update
    with pytest.raises(ValueError):
        s.decode_step(*TOKENS, bump_n_ctx=bump, fused=fused)
    assert s.n_ctx.tolist() == [7, 7] and s.r_size == 3 and not done
    refuse = False
    s.decode_step(*TOKENS, bump_n_ctx=bump, fused=fused)
    assert s.n_ctx.tolist() == [7 + bump] * 2 and s.r_size == 4 and len(done) == (3 if fused is False else 1)

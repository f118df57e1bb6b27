"""kvr_rotate_axes without a GPU: what it and make_axes refuse, and the C route beside the Python checks."""
import ctypes as C
import os

import pytest
import torch

from paper_2512_17917_amd import binding as kvr
from paper_2512_17917_amd import build as B
from tests.test_cache_fast_cpu import Fake, _both, _desc as _fake_desc, _pages as _fake_pages, _plain, _rotate_args
from tests.test_cache_ops_cpu import E, ODD, P, _desc, _pages, _rot

OK = kvr.KVR_OK


def _axes(n_axes=3, axis=None):
    a = kvr.kvr_axes(n_axes)
    for i, x in enumerate(axis if axis is not None else [i % 3 for i in range(64)]):
        a.axis[i] = x
    return a


def _turn(desc=None, rot=None, axes=None, pages=None, no_axes=False, **kw):
    a = dict(pos=P, pos_stride=2, q=P, q_stride=1536, k=P, k_stride=1536, v=P, v_stride=1536, n_rows=2, q_start=None, n_ctx=P,
             q_out=P + 16, k_out=P + 16)
    a.update(kw)
    return kvr.lib().kvr_rotate_axes(C.byref(desc or _desc()), C.byref(rot or _rot()), None if no_axes else C.byref(axes or _axes()),
                                     *a.values(), C.byref(pages) if pages else None, None)


@pytest.mark.parametrize("axes", [_axes(0), _axes(-1), _axes(9), _axes(2), _axes(3, [3]), _axes(8, [0] * 63 + [8]), _axes(8, [255])])
def test_bad_axes_are_refused(axes):
    assert _turn(axes=axes) == E


@pytest.mark.parametrize("bad", [dict(no_axes=True), dict(pos=None), dict(pos=P + 2), dict(pos_stride=-1), dict(pos_stride=(1 << 40) + 1),
                                 dict(q=None), dict(q_out=None), dict(k=None), dict(q=None, q_out=None, k=None, k_out=None),
                                 dict(q=ODD), dict(k_out=ODD), dict(q_stride=1016), dict(n_rows=-1), dict(n_rows=(1 << 27) + 1),
                                 dict(q_out=P), dict(rot=_rot(rot_dim=3)), dict(rot=_rot(inv_freq=None)), dict(rot=_rot(eps=-1.0))])
def test_bad_arguments_are_refused(bad):
    assert _turn(**bad) == E


@pytest.mark.parametrize("bad", [dict(n_rows=3), dict(n_ctx=None), dict(v=None), dict(pages=_pages(k=None)), dict(pages=_pages(page_size=0))])
def test_rows_that_go_to_pages_have_to_be_their_sequences(bad):
    a = dict(pages=_pages(), k_out=None)
    a.update(bad)
    assert _turn(**a) == E


def test_no_rows_do_nothing():
    """(Everything is looked at before, positions apart.)"""
    assert _turn(n_rows=0, pos=None, n_ctx=None) == OK
    assert _turn(n_rows=0, q_start=P, pages=_pages(), k_out=None) == OK
    assert _turn(n_rows=0, axes=_axes(9)) == E


def test_axes_past_the_turned_pairs_are_not_looked_at():
    assert _turn(rot=_rot(rot_dim=4), axes=_axes(1, [0, 0] + [7] * 62), n_rows=0) == OK
    assert _turn(rot=_rot(rot_dim=6), axes=_axes(1, [0, 0] + [7] * 62), n_rows=0) == E


def test_make_axes():
    a = kvr.make_axes([0, 2, 1])
    assert a.n_axes == 3 and list(a.axis[:4]) == [0, 2, 1, 0] and a.pairs == 3
    assert kvr.make_axes([0] * 64, 8).n_axes == 8 and kvr.make_axes([]).n_axes == 1
    for bad in (([0] * 65,), ([8],), ([-1],), ([1], 1), ([0], 9), ([0], 0)):
        with pytest.raises(ValueError):
            kvr.make_axes(*bad)


# ---------------------------------------------------------------------------
@pytest.fixture()
def fast(monkeypatch):
    if not os.path.exists(B.FAST):
        pytest.skip("the extension was left out of the build")
    real, got = kvr.lib(), []
    m = kvr._fast
    I, L, V = C.c_int32, C.c_int64, C.c_void_p
    fn = C.CFUNCTYPE(I, V, V, V, V, L, V, L, V, L, V, L, I, V, V, V, V, V, V)(lambda *a: got.append(a) or 0)
    m.setup_more(C.cast(fn, V).value, *_others(real))

    class Recorder:
        kvr_rotate_axes = staticmethod(lambda *a: got.append(tuple(_plain(x) for x in a)) or 0)

    monkeypatch.setattr(kvr, "lib", lambda: Recorder)
    monkeypatch.setattr(kvr, "_stream", lambda: 77)
    monkeypatch.setattr(kvr, "_stream_of", lambda dev: 77)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    yield got
    m.setup_more(C.cast(real.kvr_rotate_axes, V).value, *_others(real))


def _others(real):
    return [C.cast(real.kvr_attend_shared, C.c_void_p).value]


def _pos(shape=(3, 5), **kw):
    return Fake(torch.int32, shape, 0x11000, **kw)


CALLS = [dict(), dict(n_ctx=None), dict(k=None, k_out=None, v=None), dict(q=None, q_out=None), dict(n_rows=1), dict(n_rows=0)]


@pytest.mark.parametrize("case", range(len(CALLS)))
@pytest.mark.parametrize("paged", [False, True])
@pytest.mark.parametrize("pos", [_pos(), _pos((4, 9)), _pos((3, 5), strides=(0, 1))])
def test_both_routes_pass_the_same(fast, monkeypatch, case, paged, pos):
    if paged and "n_ctx" in CALLS[case]:
        return
    d = _fake_desc()
    rot = kvr.make_rotation(d, Fake(torch.float64, (64,), 0x12000))
    axes = kvr.make_axes([0] * 20 + [1] * 20 + [2] * 24)
    a = list(_rotate_args(**CALLS[case]).values())
    one, two = _both(monkeypatch, lambda: kvr.kvr_rotate_axes(d, rot, axes, pos, *a, _fake_pages(d) if paged else None), fast)
    if paged:                                     # (its pages were made anew)
        one, two = one[:17] + one[18:], two[:17] + two[18:]
    assert one == two


BAD = [(None, ValueError), (Fake(torch.int64, (3, 5), 0x11000), TypeError), (_pos((2, 5)), ValueError), (_pos((3, 4)), ValueError),
       (_pos((15,)), ValueError), (_pos((3, 5), strides=(1, 3)), ValueError), (_pos(cuda=False), ValueError),
       (Fake(torch.int32, (3, 5), 0x11000, dev=1), ValueError)]


@pytest.mark.parametrize("case", range(len(BAD)))
@pytest.mark.parametrize("route", ["C", "Python"])
def test_bad_positions_are_refused(fast, monkeypatch, case, route):
    pos, what = BAD[case]
    if route == "Python":
        monkeypatch.setattr(kvr, "_fast", None)
    d = _fake_desc()
    rot = kvr.make_rotation(d, Fake(torch.float64, (64,), 0x12000))
    with pytest.raises(what):
        kvr.kvr_rotate_axes(d, rot, kvr.make_axes([0, 1, 2, 0] * 16), pos, *_rotate_args().values())
    assert not fast


def test_axes_that_do_not_fit_the_rotation_are_refused(fast):
    d = _fake_desc()
    rot = kvr.make_rotation(d, Fake(torch.float64, (64,), 0x12000))
    for axes in (kvr.make_axes([0, 1, 2]), kvr.kvr_axes(1), None):
        with pytest.raises((ValueError, TypeError)):
            kvr.kvr_rotate_axes(d, rot, axes, _pos(), *_rotate_args().values())
    with pytest.raises(ValueError):                                # to pages, without the tokens' places
        kvr.kvr_rotate_axes(d, rot, kvr.make_axes([0] * 64), _pos(), *_rotate_args(n_ctx=None).values(), _fake_pages(d))
    assert not fast

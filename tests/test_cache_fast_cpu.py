"""The C route of kvr_rotate, kvr_attend_paged and kvr_attend_prompt takes what the Python checks take and hands back the rest.  On the CPU:
objects that answer like device tensors, and a library whose entry points only record their arguments."""
import ctypes as C
import os

import pytest
import torch

from paper_2512_17917_amd import binding as kvr
from paper_2512_17917_amd import build as B
from tests.test_fast_cpu import Fake as FlatFake

P, I, L = C.c_void_p, C.c_int32, C.c_int64


class Fake(FlatFake):
    """A device tensor of a shape and strides (dense ones if none are given)."""

    def __new__(cls, dtype, shape, at, strides=None, dev=0, cuda=True):
        n = 1
        for x in shape:
            n *= x
        dense, step = [], 1
        for x in reversed(shape):
            dense.insert(0, step)
            step *= x
        t = super().__new__(cls, dtype, n, at, cuda, strides is None)
        t._shape, t._strides, t._dev = tuple(shape), tuple(strides or dense), dev
        return t

    shape = property(lambda self: self._shape)

    def dim(self):
        return len(self._shape)

    def stride(self, i=None):
        return self._strides if i is None else self._strides[i]

    def get_device(self):
        return self._dev

    @property
    def device(self):
        return torch.device("cuda", self._dev) if self._cuda else torch.device("cpu")


@pytest.fixture()
def fast(monkeypatch):
    if not os.path.exists(B.FAST):
        pytest.skip("the extension was left out of the build")
    real = kvr.lib()
    m, got = kvr._fast, []
    rot = C.CFUNCTYPE(I, P, P, P, L, P, L, P, L, I, P, P, P, P, P, P)(lambda *a: got.append(a) or 0)
    att = C.CFUNCTYPE(I, P, P, P, P, I, I, P, P, L, P, C.c_size_t, P)(lambda *a: got.append(a) or 0)
    pro = C.CFUNCTYPE(I, P, P, I, P, P, P, I, I, P, P, L, P, C.c_size_t, P)(lambda *a: got.append(a) or 0)
    m.setup_cache(C.cast(rot, P).value, C.cast(att, P).value, C.cast(pro, P).value)

    class Recorder:
        kvr_rotate = staticmethod(lambda *a: got.append(tuple(_plain(x) for x in a)) or 0)
        kvr_attend_paged = staticmethod(lambda *a: got.append(tuple(_plain(x) for x in a)) or 0)
        kvr_attend_prompt = staticmethod(lambda *a: got.append(tuple(_plain(x) for x in a)) or 0)

    monkeypatch.setattr(kvr, "lib", lambda: Recorder)
    monkeypatch.setattr(kvr, "_stream", lambda: 77)
    monkeypatch.setattr(kvr, "_stream_of", lambda dev: 77)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    yield m, got
    m.setup_cache(*[C.cast(f, P).value for f in (real.kvr_rotate, real.kvr_attend_paged, real.kvr_attend_prompt)])


def _plain(x):
    return C.addressof(x._obj) if type(x).__name__ == "CArgObject" else x


def _desc():
    return kvr.make_desc(3, 8, 2, 1, 1, torch.bfloat16, hash_params=[(1, 2, 3, 4)])


def _rotate_args(**kw):
    bf, i32 = torch.bfloat16, torch.int32
    wide = (1536, 128, 1)
    a = dict(q=Fake(bf, (5, 8, 128), 0x1000, wide), k=Fake(bf, (5, 2, 128), 0x2000, wide), v=Fake(bf, (5, 2, 128), 0x3000, wide),
             n_rows=5, q_start=Fake(i32, (4,), 0x4000), n_ctx=Fake(i32, (3,), 0x5000), q_out=Fake(bf, (5, 8, 128), 0x6000),
             k_out=Fake(bf, (5, 2, 128), 0x7000))
    a.update(kw)
    return a


def _paged_args(**kw):
    bf = torch.bfloat16
    a = dict(q=Fake(bf, (3, 8, 128), 0x1000), n_ctx=Fake(torch.int32, (3,), 0x5000), window=5, n_sink=2,
             out=Fake(bf, (3, 8, 128), 0x6000), scores=Fake(torch.float32, (3, 2, 40), 0x7000), n_cap=40,
             ws=Fake(torch.uint8, (999,), 0x8000))
    a.update(kw)
    return a


def _pages(d):
    bf = torch.bfloat16
    return kvr.make_pages(d, Fake(bf, (9, 2, 16, 128), 0x9000), Fake(bf, (9, 2, 16, 128), 0xa000), Fake(torch.int32, (3, 4), 0xb000))


def _both(monkeypatch, call, got):
    """What reached the library by the C route and by Python's checks."""
    call()
    monkeypatch.setattr(kvr, "_fast", None)
    call()
    assert len(got) == 2
    norm = [tuple(x.value if hasattr(x, "value") else x for x in a) for a in got]
    return norm


GOOD_ROTATE = [dict(), dict(q_start=None, n_rows=3), dict(k=None, k_out=None, v=None), dict(q=None, q_out=None), dict(v=None),
               dict(n_rows=1), dict(n_rows=0)]


@pytest.mark.parametrize("case", range(len(GOOD_ROTATE)))
@pytest.mark.parametrize("paged", [False, True])
def test_rotate_both_routes_pass_the_same(fast, monkeypatch, case, paged):
    m, got = fast
    d = _desc()
    rot = kvr.make_rotation(d)
    pages = _pages(d) if paged else None
    a = _rotate_args(**GOOD_ROTATE[case])
    one, two = _both(monkeypatch, lambda: kvr.kvr_rotate(d, rot, *a.values(), pages), got)
    assert one == two


def test_paged_both_routes_pass_the_same(fast, monkeypatch):
    m, got = fast
    d = _desc()
    pages = _pages(d)
    for kw in (dict(), dict(scores=None, n_cap=0), dict(ws=None)):
        del got[:]
        a = list(_paged_args(**kw).values())
        with monkeypatch.context() as p:
            one, two = _both(p, lambda: kvr.kvr_attend_paged(d, *a[:2], pages, *a[2:]), got)
        assert one == two


BAD_ROTATE = [dict(q=Fake(torch.float32, (5, 8, 128), 1)), dict(q=Fake(torch.bfloat16, (4, 8, 128), 1)),
              dict(k=Fake(torch.bfloat16, (5, 8, 128), 1)), dict(q=Fake(torch.bfloat16, (5, 1024), 1)),
              dict(q=Fake(torch.bfloat16, (5, 8, 128), 1, (1024, 1, 8))), dict(v=Fake(torch.bfloat16, (5, 2, 128), 1, cuda=False)),
              dict(q=Fake(torch.bfloat16, (5, 8, 128), 1, dev=1)), dict(n_ctx=Fake(torch.int32, (2,), 1)), dict(n_ctx=None),
              dict(n_ctx=Fake(torch.int64, (3,), 1)), dict(q_start=Fake(torch.int32, (3,), 1)),
              dict(q_out=Fake(torch.bfloat16, (5, 8, 127), 1)), dict(q_out=Fake(torch.bfloat16, (5, 8, 128), 1, (1536, 128, 1))),
              dict(k_out=Fake(torch.bfloat16, (5, 2, 128), 1, dev=1)), dict(q=5)]


@pytest.mark.parametrize("case", range(len(BAD_ROTATE)))
def test_rotate_refusals(fast, monkeypatch, case):
    m, got = fast
    d = _desc()
    rot = kvr.make_rotation(d)
    a = _rotate_args(**BAD_ROTATE[case])
    assert m.rotate(C.addressof(d), C.addressof(rot), 0, 0, 77, *a.values()) is None and not got
    with pytest.raises((TypeError, ValueError)):
        kvr.kvr_rotate(d, rot, *a.values())
    assert not got


BAD_PAGED = [dict(q=Fake(torch.bfloat16, (3, 8, 127), 1)), dict(out=Fake(torch.float32, (3, 8, 128), 1)), dict(n_ctx=None),
             dict(scores=Fake(torch.float32, (3, 2, 39), 1)), dict(out=Fake(torch.bfloat16, (3, 8, 128), 1, dev=2)),
             dict(ws=Fake(torch.uint8, (9,), 1, (2,))), dict(scores=Fake(torch.bfloat16, (3, 2, 40), 1))]


@pytest.mark.parametrize("case", range(len(BAD_PAGED)))
def test_paged_refusals(fast, case):
    m, got = fast
    d = _desc()
    pages = _pages(d)
    a = list(_paged_args(**BAD_PAGED[case]).values())
    assert m.attend_paged(C.addressof(d), C.addressof(pages), 0, 77, *a) is None and not got
    with pytest.raises((TypeError, ValueError)):
        kvr.kvr_attend_paged(d, *a[:2], pages, *a[2:])
    assert not got


def _prompt_args(**kw):
    bf, i32 = torch.bfloat16, torch.int32
    a = dict(q=Fake(bf, (7, 8, 128), 0x1000), n_rows=7, q_start=Fake(i32, (4,), 0x4000), n_ctx=Fake(i32, (3,), 0x5000), window=5,
             n_sink=2, out=Fake(bf, (7, 8, 128), 0x6000), scores=Fake(torch.float32, (3, 2, 40), 0x7000), n_cap=40,
             ws=Fake(torch.uint8, (999,), 0x8000))
    a.update(kw)
    return a


def test_prompt_both_routes_pass_the_same(fast, monkeypatch):
    m, got = fast
    d = _desc()
    pages = _pages(d)
    for kw in (dict(), dict(scores=None, n_cap=0), dict(ws=None), dict(q_start=None, n_rows=3), dict(n_rows=0)):
        del got[:]
        a = list(_prompt_args(**kw).values())
        with monkeypatch.context() as p:
            one, two = _both(p, lambda: kvr.kvr_attend_prompt(d, *a[:4], pages, *a[4:]), got)
        assert one == two


BAD_PROMPT = [dict(q=Fake(torch.bfloat16, (6, 8, 128), 1)), dict(out=Fake(torch.float32, (7, 8, 128), 1)), dict(n_ctx=None),
              dict(q_start=Fake(torch.int32, (3,), 1)), dict(scores=Fake(torch.float32, (3, 2, 39), 1)),
              dict(q_start=Fake(torch.int32, (4,), 1, dev=1)), dict(ws=Fake(torch.uint8, (9,), 1, dev=1)), dict(q=None)]


@pytest.mark.parametrize("case", range(len(BAD_PROMPT)))
def test_prompt_refusals(fast, case):
    m, got = fast
    d = _desc()
    pages = _pages(d)
    a = list(_prompt_args(**BAD_PROMPT[case]).values())
    assert m.attend_prompt(C.addressof(d), C.addressof(pages), 0, 77, *a) is None and not got
    with pytest.raises((TypeError, ValueError)):
        kvr.kvr_attend_prompt(d, *a[:4], pages, *a[4:])
    assert not got


def test_another_device_is_refused(fast, monkeypatch):
    """Pages, weights or frequencies of one device in a call on another; tensors of two devices in one struct."""
    m, got = fast
    d = _desc()
    pages, a = _pages(d), list(_paged_args().values())
    inv = Fake(torch.float64, (64,), 0xc000)
    rot = kvr.make_rotation(d, inv)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 1)
    with pytest.raises(ValueError):
        kvr.kvr_attend_paged(d, *a[:2], pages, *a[2:])
    with pytest.raises(ValueError):
        kvr.kvr_rotate(d, rot, *_rotate_args().values())
    with pytest.raises(ValueError):
        kvr.make_rotation(d, inv, q_weight=Fake(torch.bfloat16, (128,), 1, dev=1))
    assert not got


def test_pages_of_another_descriptor(fast):
    d = _desc()
    pages = _pages(d)
    a = list(_paged_args().values())
    for other in (kvr.make_desc(4, 8, 2, 1, 1, torch.bfloat16, hash_params=[(1, 2, 3, 4)]),
                  kvr.make_desc(3, 8, 4, 1, 1, torch.bfloat16, hash_params=[(1, 2, 3, 4)]),
                  kvr.make_desc(3, 8, 2, 1, 1, torch.float32, hash_params=[(1, 2, 3, 4)])):
        with pytest.raises(ValueError):
            kvr.kvr_attend_paged(other, *a[:2], pages, *a[2:])

"""PagedCache.share with lists, on the CPU: they go to tensors of the cache's own, at the same address for every call, so that a step
captured with lists does not read memory that a later share() has given back."""
import pytest
import torch

from paper_2512_17917_amd import binding as kvr
from paper_2512_17917_amd.state import PagedCache

B = 5


@pytest.fixture()
def cache(monkeypatch):
    def make(start, n_shared):
        g = kvr.kvr_groups(start.data_ptr(), n_shared.data_ptr(), n_shared.numel())
        g.tensors = (start, n_shared)
        return g
    monkeypatch.setattr(kvr, "make_groups", make)
    monkeypatch.setattr(PagedCache, "_room_to_share", lambda self, groups, rows: torch.empty(256, dtype=torch.uint8))
    c = PagedCache.__new__(PagedCache)
    c.desc, c.device = kvr.make_desc(B, 8, 2, 1, 1, torch.bfloat16), torch.device("cpu")
    c.groups = c.lists = c.ws_shared = None
    return c


def _held(g):
    return [t.tolist() for t in g.tensors]


def _groups(g):
    """Sequences of each group with something in common, as the kernels read them."""
    start, common = ([min(max(x, 0), B) for x in t] if i == 0 else t for i, t in enumerate(_held(g)))
    return [(a, b, c) for a, b, c in zip(start, start[1:], common) if c and b > a]


def test_lists_stay_where_they_are(cache):
    cache.share([0, 3], [7])
    first, at = cache.groups, [t.data_ptr() for t in cache.groups.tensors]
    assert _groups(first) == [(0, 3, 7)]
    for start, common, want in (([0, 2, 5], [4, 9], [(0, 2, 4), (2, 5, 9)]), ([1, 1, 4, 4], [3, 6, 8], [(1, 4, 6)]),
                                (list(range(B + 1)), [1] * B, [(b, b + 1, 1) for b in range(B)]), ([-3, 99], [2], [(0, B, 2)]),
                                ((0, 3, 5, 5), (7, 0), [(0, 3, 7)])):
        cache.share(start, common)
        assert cache.groups is first and first.n_groups == B
        assert [t.data_ptr() for t in cache.groups.tensors] == at and [first.start, first.n_shared] == at
        assert _groups(first) == want
        starts = _held(first)[0]
        assert all(min(max(x, 0), B) <= min(max(y, 0), B) for x, y in zip(starts, starts[1:]))


@pytest.mark.parametrize("end", [(None, None), ([], []), ([0], []), "tensors"])
def test_what_ends_them_leaves_none_for_a_captured_step(cache, end):
    cache.share([0, 3], [7])
    first = cache.groups
    if end == "tensors":
        end = torch.tensor([0, 5], dtype=torch.int32), torch.tensor([6], dtype=torch.int32)
        cache.share(*end)
        assert cache.groups is not first and cache.groups.tensors[0] is end[0]
    else:
        cache.share(*end)
        assert cache.groups is None
    assert _groups(first) == []
    cache.share([2, 4], [5])
    assert cache.groups is first and _groups(first) == [(2, 4, 5)]


@pytest.mark.parametrize("start,common", [([0], [5]), ([0, 3], [5, 6]), ([0, 3, 2], [5, 6]), (list(range(B + 2)), [1] * (B + 1))])
def test_lists_that_cannot_be_are_refused_and_change_nothing(cache, start, common):
    cache.share([0, 3], [7])
    first, held = cache.groups, _held(cache.groups)
    with pytest.raises(ValueError):
        cache.share(start, common)
    assert cache.groups is first and _held(first) == held

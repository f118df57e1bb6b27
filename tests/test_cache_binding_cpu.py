"""What the binding and the cache's classes refuse, on the CPU: calls that would read past an operand, mix up tokens or drop scores."""
import pytest
import torch

from paper_2512_17917_amd import binding as kvr
from paper_2512_17917_amd.state import LayerState, PagedCache
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


def _cache_of(table, n_ctx, n_pages=5, page=4):
    """A PagedCache on the CPU, of which `dense` alone is called."""
    c = PagedCache.__new__(PagedCache)
    c.desc = _desc()
    c.desc.batch = len(table)
    c.k, c.v = torch.randn(2, n_pages, 2, page, 8)
    c.table, c.n_ctx = torch.tensor(table, dtype=torch.int32), torch.tensor(n_ctx, dtype=torch.int32)
    return c


def test_dense_takes_tokens_that_are_there():
    c = _cache_of([[3, 0, -1], [4, 1, 9]], [7, 8])
    for n in (1, 4, 5, 7):
        for got, pool in zip(c.dense(n), (c.k, c.v)):
            for b, pages in enumerate(([3, 0], [4, 1])):
                assert torch.equal(got[b], torch.cat([pool[p] for p in pages], 1)[:, :n]), n


@pytest.mark.parametrize("table,n_ctx,n", [([[3, -1, 2], [4, 1, 0]], [9, 9], 5),       # no page: not the pool's last one
                                           ([[3, 1, 2], [4, 5, 0]], [9, 9], 5),        # past the pool
                                           ([[3, 1, 2], [4, 0, 0]], [9, 4], 5),        # tokens that have not come yet
                                           ([[3, 1], [4, 0]], [8, 8], 9),              # more than the table holds
                                           ([[3, 1], [4, 0]], [8, 8], 0), ([[3, 1], [4, 0]], [8, 8], -1)])
def test_dense_refuses_tokens_that_are_not(table, n_ctx, n):
    with pytest.raises(ValueError):
        _cache_of(table, n_ctx).dense(n)


def _no_device(monkeypatch):
    """The calls into the library record themselves; tensors may live anywhere."""
    calls = []
    for name in ("kvr_attend_prompt", "kvr_attend_paged", "kvr_rotate", "kvr_attend_decode"):
        monkeypatch.setattr(kvr, name, lambda *a, _n=name: calls.append(_n))
    for name in ("kvr_attend_prompt_workspace_size", "kvr_attend_paged_workspace_size"):
        monkeypatch.setattr(kvr, name, lambda *a: 0)
    monkeypatch.setattr(kvr, "make_pages", lambda *a: None)
    monkeypatch.setattr(kvr, "alloc_workspace", lambda *a: torch.empty(256, dtype=torch.uint8))
    return calls


@pytest.mark.parametrize("shape", [(2, 8, 8, 128), (2, 10, 8, 128), (1, 9, 8, 128), (3, 9, 8, 128), (2, 9, 4, 128), (18, 8, 128)])
def test_a_prompt_has_a_query_for_each_of_its_tokens(monkeypatch, shape):
    """Fewer rows would be taken for the newest tokens', more for tokens before the first: from_prefill's scores would lack them."""
    calls = _no_device(monkeypatch)
    d = kvr.make_desc(2, 8, 2, 3, 5, torch.bfloat16, seed=1)
    K, V = torch.zeros(2, 2, 2, 9, 128, dtype=torch.bfloat16)
    q = torch.zeros(shape, dtype=torch.bfloat16)
    with pytest.raises(ValueError):
        LayerState.from_prefill(d, K, V, None, n_recent=4, k_candidate=2, max_new_tokens=1, q_prompt=q)
    assert not calls


def test_a_given_table_has_the_width_that_it_is_said_to_have(monkeypatch):
    """With more columns than table_cap, tokens past table_cap * page_size would be attended but their scores dropped."""
    _no_device(monkeypatch)
    d = kvr.make_desc(2, 8, 2, 3, 5, torch.bfloat16, seed=1)
    make = lambda table, **kw: PagedCache(d, n_pages=4, page_size=16, table_cap=6, device="cpu", table=table, **kw)
    monkeypatch.setattr(kvr, "make_rotation", lambda *a: None)
    for cols in (5, 7):
        with pytest.raises(ValueError):
            make(torch.zeros(2, cols, dtype=torch.int32))
    for rows in (2, 3):
        c = make(torch.zeros(rows, 6, dtype=torch.int32))
        assert c.scores.shape == (2, 2, 96)
    assert make(None).table.shape == (2, 6)


@pytest.mark.parametrize("first,pages", [(6, [3]), (5, [1, 2]), (-1, [3]), (-2, [1, 2]), (7, [3])])
def test_pages_past_the_table_are_refused(first, pages):
    """One page just past the end was assigned nowhere, without a word."""
    c = _cache_of([[-1] * 6, [-1] * 6], [0, 0])
    c.device = torch.device("cpu")
    with pytest.raises(ValueError):
        c.assign(1, first, pages)
    assert bool((c.table == -1).all())
    c.assign(1, 4, [2, 0])
    c.assign(0, 6, [])
    assert c.table.tolist() == [[-1] * 6, [-1] * 4 + [2, 0]]

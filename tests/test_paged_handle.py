"""KVCache on the CPU, with the checks that need device memory put aside: what it remembers
of its tensors after the first call."""
import copy
import pickle

import pytest

torch = pytest.importorskip("torch")
ce = pytest.importorskip("paper_2608_29291_amd")


@pytest.fixture
def cache(monkeypatch):
    monkeypatch.setattr(ce, "_device", lambda: -1)
    monkeypatch.setattr(ce, "_chk", lambda t, *a: t.data_ptr())
    monkeypatch.setattr(ce, "_chk_strided", lambda t, *a: t.data_ptr())
    pool = torch.zeros(12, 2, 2, 16, 128, dtype=torch.bfloat16)  # keys and values of a layer side by side
    return ce.KVCache(pool[:, 0], pool[:, 1], torch.zeros(6, 4, dtype=torch.int32))


def test_it_is_looked_over_once(cache):
    assert cache.c() is cache.c()


@pytest.mark.parametrize("change,field,value", [
    (lambda c: c.page_table.resize_(3, 4), "B", 3),
    (lambda c: c.page_table.resize_(4, 6), "max_pages", 6),
    (lambda c: [x.as_strided_((5, *x.shape[1:]), x.stride()) for x in (c.k, c.v)], "n_pages", 5),
])
def test_a_change_in_place_is_seen(cache, change, field, value):
    first = cache.c()
    assert getattr(first, field) != value
    change(cache)
    assert getattr(cache.c(), field) == value


def test_a_change_of_stride_alone_is_seen(cache):
    assert cache.c().page_stride == 2 * 2 * 16 * 128
    for x in (cache.k, cache.v):
        x.as_strided_((3, *x.shape[1:]), x.stride())
    cache.c()
    for x in (cache.k, cache.v):
        x.as_strided_(x.shape, (4 * 2 * 16 * 128, *x.stride()[1:]))
    assert cache.c().page_stride == 4 * 2 * 16 * 128


def test_a_change_of_type_is_seen(cache):
    cache.c()
    for x in (cache.k, cache.v):
        x.data = x.view(torch.float8_e4m3fn)[..., :128].as_strided(x.shape, [2 * s for s in x.stride()[:-1]] + [1])
    assert cache.c().dtype == ce.CE_E4M3


def test_a_used_handle_is_copied_and_pickled(cache):
    cache.c()
    for other in (copy.copy(cache), copy.deepcopy(cache), pickle.loads(pickle.dumps(cache))):
        assert other.k_scale is None and torch.equal(other.page_table, cache.page_table)
        assert other.k.stride() == cache.k.stride() and other.c().k == other.k.data_ptr()
        other.page_table.resize_(2, 4)
        assert other.c().B == 2 and (cache.c().B == 6 or other.page_table is cache.page_table)
        other.page_table.resize_(6, 4)

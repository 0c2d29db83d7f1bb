"""State that outlives a call of the paged cache: page numbers that go back on the free
stack, and a handle whose tensors change in place, is copied or pickled after its first call."""
import copy
import pickle

import numpy as np
import pytest

import paged_util as U

pytestmark = pytest.mark.gpu


def i32(x):
    import torch
    return torch.tensor(x, dtype=torch.int32).cuda()


@pytest.mark.parametrize("B", [2, 1500])
@pytest.mark.parametrize("bad", [-1, 8, 1 << 30])
def test_page_numbers_out_of_range_are_reported_when_they_go_back(bad, B):
    """A length past what the row of the table holds: the call that pushes the entry says so, and
    the one that pops it again; its rows get no slot."""
    import torch
    import paper_2608_29291_amd as ce
    kv = torch.empty(8, 1, 16, U.DH, dtype=torch.bfloat16, device="cuda")
    table = torch.full((B, 3), -9, dtype=torch.int32, device="cuda")
    table[B - 1, :2] = i32([5, bad])
    c = ce.KVCache(kv, kv, table)
    lens, reset = torch.zeros(B, dtype=torch.int32, device="cuda"), torch.zeros(B, dtype=torch.uint8, device="cuda")
    lens[B - 1], reset[B - 1] = 20, 1
    free, count, start, status = i32([7, 6, 0, 0, 0, 0, 0, 0]), i32([2]), torch.zeros_like(lens), i32([77])
    ce.ce_kv_reserve(c, lens, None, free, count, start, None, reset=reset, status=status)
    assert count.item() == 4 and free[:4].tolist() == [7, 6, 5, bad] and not lens.any()
    assert status.item() == ce.CE_DEV_BAD_CACHE
    # the first sequence pops it
    off = torch.full((B + 1,), 20, dtype=torch.int32, device="cuda")
    off[0] = 0
    slots = torch.full((20,), 9, dtype=torch.int32, device="cuda")
    ce.ce_kv_reserve(c, lens, off, free, count, start, slots, status=status)
    assert status.item() == ce.CE_DEV_BAD_CACHE and count.item() == 2 and lens[0].item() == 20
    assert slots.tolist() == [-1] * 16 + [5 * 16 + i for i in range(4)]
    # pages in order go back without a word
    table[0, :2] = i32([5, 4])
    reset[0] = 1
    ce.ce_kv_reserve(c, lens, None, free, count, start, None, reset=reset, status=status)
    assert status.item() == 0 and free[:4].tolist() == [7, 6, 5, 4]


def attend(c, p, q, lens):
    import torch
    import paper_2608_29291_amd as ce
    qd = torch.from_numpy(q).to(torch.bfloat16).cuda()
    o = torch.empty_like(qd)
    ce.ce_paged_attention(c, qd, o, torch.arange(len(q) + 1, dtype=torch.int32, device="cuda"), i32(lens), True, U.DH ** -0.5)
    return o.float().cpu().numpy()


def test_a_table_that_changes_in_place_is_seen():
    """Same memory, other rows: the next call takes the table as it is now."""
    p = U.Paged([40, 33, 50, 20], 2, 16, "bf16", seed=5, extra_cols=0)
    q = U.bf16(np.random.default_rng(1).standard_normal((4, 4, U.DH)))
    c = p.cache()
    U.check(attend(c, p, q, p.lens), *p.answer(q, [1] * 4, True, U.DH ** -0.5))
    c.page_table.resize_(2, 4)
    assert c.c().B == 2 and c.c().max_pages == 4
    c.page_table.resize_(4, 4)
    U.check(attend(c, p, q, p.lens), *p.answer(q, [1] * 4, True, U.DH ** -0.5))
    c.page_table.t_()
    with pytest.raises(ValueError, match="page_table"):
        attend(c, p, q, p.lens)
    c.page_table.t_()
    c.k.resize_(p.n_pages - 1, 2, 16, U.DH)
    with pytest.raises(ValueError, match="one shape"):
        attend(c, p, q, p.lens)
    c.v.resize_(p.n_pages - 1, 2, 16, U.DH)
    assert c.c().n_pages == p.n_pages - 1


@pytest.mark.parametrize("dtype", ["bf16", "e4m3"])
def test_a_used_cache_is_copied_and_pickled(dtype):
    p = U.Paged([700, 33], 2, 16, dtype, seed=6)
    q = U.bf16(np.random.default_rng(1).standard_normal((2, 4, U.DH)))
    c = p.cache()
    want = attend(c, p, q, p.lens)
    others = [copy.copy(c), copy.deepcopy(c)]
    if dtype == "bf16":  # (pickle.loads fails on any float8 tensor: torch's own limit)
        others.append(pickle.loads(pickle.dumps(c)))
    for other in others:
        assert np.array_equal(attend(other, p, q, p.lens), want)
    deep = copy.deepcopy(c)
    deep.v.zero_()  # pages of its own
    assert not attend(deep, p, q, p.lens).any() and np.array_equal(attend(c, p, q, p.lens), want)

"""State that outlives a call of the paged cache: page numbers that go back on the free
stack."""
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

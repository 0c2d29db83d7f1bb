"""Accepted rows in the paged cache, lengths and pages that go back."""
import numpy as np
import pytest
import torch

import draft_util as du
import paged_util as pu
from oracle import draft as od

pytestmark = pytest.mark.gpu
ce = pytest.importorskip("paper_2608_29291_amd")


def rows_of(p, cache, b):
    """A sequence's stored keys and values, as bytes."""
    out = []
    for pool in (cache.k, cache.v):
        x = pool.view(torch.uint8).cpu().numpy().reshape(p.n_pages, p.hkv, p.page, -1)
        out.append([x[p.table[b, j // p.page], :, j % p.page].tobytes() for j in range(p.lens[b])])
    return out


def run(p, new, kept, start=None, n_kept=None, rows=None):
    c = p.cache()
    before = [rows_of(p, c, b) for b in range(len(new))]
    start = [m - n for m, n in zip(p.lens, new)] if start is None else start
    flat = [x for n, k in zip(new, kept) for x in list(k)[:n] + [-1] * (n - len(k))]
    flat = np.array(flat + [0, 1], np.int32)
    n_kept = [len(k) for k in kept] if n_kept is None else n_kept
    free = [p.free.copy()]
    k0, v0 = c.k.clone(), c.v.clone()
    ce.ce_kv_keep(c, du.up(du.offsets(new)), du.up(np.array(start, np.int32)), du.up(flat), du.up(np.array(n_kept, np.int32)))
    touched = 0
    for b in range(len(new)):
        got = rows_of(p, c, b)
        for x, y in zip(before[b], got):
            want = x if start[b] < 0 else od.keep(x, start[b], kept[b][:new[b]][:max(n_kept[b], 0)])
            assert y == want, b
            touched += sum(a != w for a, w in zip(x, want))
    changed = sum(int((a.view(torch.uint8).view(p.n_pages, p.hkv, p.page, -1) !=
                       d.view(torch.uint8).view(p.n_pages, p.hkv, p.page, -1)).any(-1).any(1).sum())
                  for a, d in ((k0, c.k), (v0, c.v)))
    assert changed <= touched, "other rows were written"


@pytest.mark.parametrize("dtype", ["bf16", "e4m3"])
@pytest.mark.parametrize("page,hkv", [(16, 1), (32, 4), (64, 2), (256, 20)])
def test_keep(dtype, page, hkv):
    rng = np.random.default_rng(page)
    new = [1, 33, 64, 0, 20, 40, 7]
    lens = [n + m for n, m in zip(new, [0, 15, 31, 5, 1000, 600, 250])]
    kept = [[0] + sorted(rng.choice(np.arange(1, n), min(n - 1, k), replace=False).tolist()) if n else []
            for n, k in zip(new, [3, 5, 30, 2, 1, 39, 0])]
    run(pu.Paged(lens, hkv, page, dtype, poison=1.0), new, kept)


def test_keep_edges():
    p = pu.Paged([40, 50, 60, 70, 20, 30], 2, 16, "bf16", poison=1.0)
    new = [10, 10, 10, 10, 10, 10]
    kept = [[0, 3, 3, 9], [0, 9, 5], [0, 10, 11], [-1, 2], list(range(10)), [2, 4, 6, 8]]
    # rows that do not rise or are none end the list; a sequence without a start, counts out of range
    run(p, new, kept, start=[30, 40, 50, 60, -1, 20], n_kept=[4, 3, 3, 2, 10, 99])
    run(p, new, kept, n_kept=[0, -4, 1, 2, 10, 4])


def test_keep_skips_pages_that_are_none():
    p = pu.Paged([64], 1, 16, "bf16", poison=1.0)
    c = p.cache()
    c.page_table[0, 2] = 1 << 20  # tokens 32 .. 47
    k0 = c.k.clone()
    start, kept = 20, [0, 15, 30, 40]  # to 21 .. 23 from 35 (on no page), 50, 60
    ce.ce_kv_keep(c, du.up(du.offsets([44])), du.up(np.array([start], np.int32)), du.up(np.array(kept + [0] * 40, np.int32)),
                  du.up(np.array([4], np.int32)))
    at = lambda j: (int(p.table[0, j // 16]), j % 16)
    for j, src in ((21, 21), (22, 50), (23, 60)):
        assert torch.equal(c.k[at(j)[0], :, at(j)[1]], k0[at(src)[0], :, at(src)[1]]), j


def test_keep_of_layers_that_share_an_allocation():
    p = pu.Paged([100, 60], 2, 16, "bf16", poison=1.0)
    c = p.cache()
    pool = torch.zeros((p.n_pages, 3, 2, 16, 128), dtype=torch.bfloat16, device="cuda")
    pool[:, 1] = c.k
    pv = torch.zeros_like(pool)
    pv[:, 1] = c.v
    d = ce.KVCache(pool[:, 1], pv[:, 1], c.page_table)
    args = (du.up(du.offsets([50, 20])), du.up(np.array([50, 40], np.int32)),
            du.up(np.array([0, 7, 30, 49] + [-1] * 46 + [0, 1, 19] + [-1] * 17, np.int32)), du.up(np.array([4, 3], np.int32)))
    ce.ce_kv_keep(c, *args)
    ce.ce_kv_keep(d, *args)
    assert torch.equal(pool[:, 1], c.k) and torch.equal(pv[:, 1], c.v)
    assert (pool[:, ::2] == 0).all() and (pv[:, ::2] == 0).all()


def trim(p, lens, start, n_kept, room=None, count=None, in_place=False):
    c = p.cache()
    stack = np.full(p.n_pages, -5, np.int32)
    stack[:len(p.free)] = p.free
    count = len(p.free) if count is None else count
    t = lambda x: du.up(np.array(x, np.int32))
    free, cnt, ln = t(stack), t([count]), t(lens)
    out = ln if in_place else t([-9] * len(lens))
    cnt_out = cnt if in_place else t([-9])
    st = t([-1])
    ce.ce_kv_trim(c, ln, t(start), t(n_kept), free, cnt, lens_out=None if in_place else out,
                  free_count_out=None if in_place else cnt_out, status=st)
    return out.tolist(), free.tolist(), int(cnt_out), int(st), stack.tolist()


@pytest.mark.parametrize("page", [16, 128])
@pytest.mark.parametrize("B", [1, 7, 1500])
@pytest.mark.parametrize("in_place", [False, True])
def test_trim(page, B, in_place):
    rng = np.random.default_rng(B)
    new = rng.integers(0, 200, B).tolist()
    lens = [n + int(m) for n, m in zip(new, rng.integers(0, 300, B))]
    start = [m - n if rng.random() < 0.9 else -1 for m, n in zip(lens, new)]
    kept = [int(rng.integers(0, n + 1)) for n in new]
    p = pu.Paged([0] * B, 1, page, "bf16", spare=4, extra_cols=40)
    held = [-(-m // page) for m in lens]
    # (a table of its own: the pages that the lengths need, and four free ones)
    p.n_pages = sum(held) + 4
    order = rng.permutation(p.n_pages)
    p.table = np.full((B, 40), 1 << 30, np.int32)
    at = 0
    for b, h in enumerate(held):
        p.table[b, :h] = order[at:at + h]
        at += h
    p.free = order[at:].astype(np.int32)
    p.pk = p.pv = torch.zeros((p.n_pages, 1, page, 128), dtype=torch.bfloat16)
    want_free, want_lens = p.free.tolist(), []
    for b in range(B):
        now = lens[b] if start[b] < 0 else start[b] + kept[b]
        want_free += p.table[b, -(-now // page):held[b]].tolist()
        want_lens.append(now)
    got, free, count, st, _ = trim(p, lens, start, kept, in_place=in_place)
    assert got == want_lens and count == len(want_free) and free[:count] == want_free and st == 0


def test_trim_of_numbers_out_of_range():
    p = pu.Paged([100, 40, 33], 1, 16, "bf16", spare=3)
    # a length past the table's row is clamped, a count past the pool too; more kept than there are
    most = p.width * 16
    got, _, count, st, _ = trim(p, [1 << 30, 40, 33], [-1, 20, 30], [0, 50, -2])
    assert got == [most, 40, 30] and count == 3 + 1 and st == ce.CE_DEV_BAD_CACHE
    # a full stack takes no more; nothing is written behind it
    got, free, count, st, _ = trim(p, [100, 40, 33], [0, 0, 0], [0, 0, 0], count=p.n_pages)
    assert got == [0, 0, 0] and count == p.n_pages and st == ce.CE_DEV_BAD_CACHE
    # a page number that is none is pushed, and reported
    p.table[0, 1] = -3
    _, free, count, st, _ = trim(p, [20, 0, 0], [0, 0, 0], [16, 0, 0])
    assert st == ce.CE_DEV_BAD_CACHE and free[count - 1] == -3

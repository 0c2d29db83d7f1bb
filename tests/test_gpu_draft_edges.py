"""Drafted decoding where its arguments end: offsets out of order, long sequences, large batches."""
import numpy as np
import pytest
import torch

import draft_util as du
import paged_util as pu
from oracle import draft as od
from test_gpu_verify import Case

pytestmark = pytest.mark.gpu
ce = pytest.importorskip("paper_2608_29291_amd")


@pytest.mark.parametrize("drawn", [False, True])
@pytest.mark.parametrize("off", [[0, 25, 5, 30], [-3, 10, 20, 1 << 30], [7, 7, 7, 7], [30, 20, 10, 0], [0, 30, 10, 30]])
def test_every_sequence_gets_a_count_and_a_token_whatever_the_offsets(off, drawn):
    # the calls behind this one take lengths from the count: it must not be what the memory held before
    c = Case([10, 10, 10], 500, torch.float32, drawn=drawn)
    c.off = np.array(off, np.int32)
    for pad in (3, 5000):
        for fill in (0xff, 0):
            _, n_kept, following = c.run(rest=False, pad=pad, fill=fill)  # (filled with -9 before)
            assert all(0 <= k <= 30 + pad for k in n_kept), n_kept
            assert all(-1 <= t < 500 for t in following), following
            ends = np.clip(c.off, 0, 30 + pad)
            assert all(k == 0 and t == -1 for k, t, lo, hi in zip(n_kept, following, ends, ends[1:]) if hi <= lo)


def long_tree(rng, n, kind):
    """Parents of n rows, far more than LDS holds."""
    i = np.arange(n)
    if kind == "near":  # deep, with side branches
        p = i - 1 - rng.integers(0, 3, n)
    elif kind == "far":  # parents anywhere before, a few of them far away
        p = (i * rng.random(n)).astype(int)
    else:  # chains that begin again, at no parent, every few thousand rows
        p = np.where(rng.random(n) < 3e-4, -1, i - 1)
    p = np.where(p < 0, -1, p)
    p[0] = -1
    return p.tolist()


def plain_masks(parents, words):
    """Words and depths, a row at a time, a mask as one whole number."""
    cut, seen, depth = (1 << 32 * words) - 1, [], []
    for i, p in enumerate(parents):
        own = 1 << i if i < 32 * words else 0
        good = 0 <= p < i
        seen.append((seen[p] if good else 0) | own & cut)
        depth.append(depth[p] + 1 if good else 0)
    m = np.frombuffer(b"".join(s.to_bytes(4 * words, "little") for s in seen), np.uint32).reshape(-1, words)
    return m, np.array(depth)


def run_masks(new, parents, words, base, rows, with_mask=True, with_positions=True):
    off = du.up(du.offsets(new))
    d = ce.Drafts(off, rows=rows) if parents is None else ce.Drafts(off, du.up(np.array(parents + [0] * (rows - sum(new)), np.int32)))
    mask = torch.full((rows, words), 0x55555555, dtype=torch.int32, device="cuda") if with_mask else None
    pos = torch.full((rows,), -7, dtype=torch.int32, device="cuda") if with_positions else None
    ce.ce_draft_masks(d, mask, positions=pos, base=du.up(np.array(base, np.int32)))
    return (mask.cpu().numpy().view(np.uint32) if with_mask else None), (pos.cpu().numpy() if with_positions else None)


@pytest.mark.parametrize("kind", ["near", "far", "chains"])
@pytest.mark.parametrize("words", [1, 3, 64])
@pytest.mark.parametrize("n", [8192, 8193, 10240, 10241, 30011])
def test_masks_of_long_sequences(n, words, kind):
    rng = np.random.default_rng(n + words)
    new = [5, n, 0, 33]
    trees = [du.tree(rng, 5), long_tree(rng, n, kind), [], du.tree(rng, 33)]
    rows, base = sum(new) + 3, [7, 2 ** 31 - 100, 1, -5]
    mask, pos = run_masks(new, sum(trees, []), words, base, rows)
    at = 0
    for t, b in zip(trees, base):
        if t:
            m, depth = plain_masks(t, words)
            np.testing.assert_array_equal(mask[at:at + len(t)], m)
            np.testing.assert_array_equal(pos[at:at + len(t)], (depth + b).astype(np.uint32).view(np.int32))  # (modulo 2^32)
        at += len(t)
    assert (mask[at:] == 0x55555555).all() and (pos[at:] == -7).all(), "rows behind the last were written"
    np.testing.assert_array_equal(run_masks(new, sum(trees, []), words, base, rows, with_positions=False)[0], mask)
    np.testing.assert_array_equal(run_masks(new, sum(trees, []), words, base, rows, with_mask=False)[1], pos)


@pytest.mark.parametrize("parents", [False, True])
def test_a_chain_of_a_million_rows_takes_no_walk_to_its_root(parents):
    n = 1 << 20
    args = [n, 4], (list(range(-1, n - 1)) + [-1, 0, 0, 1] if parents else None), 2, [3, 9], n + 4
    run_masks(*args)
    torch.cuda.synchronize()
    a, b = (torch.cuda.Event(enable_timing=True) for _ in range(2))
    a.record()
    mask, pos = run_masks(*args)
    b.record()
    torch.cuda.synchronize()
    # 2^39 steps of such walks, 1024 at a time, take minutes
    assert a.elapsed_time(b) < 5000
    np.testing.assert_array_equal(pos, np.concatenate([np.arange(n) + 3, [9, 10, 10, 11] if parents else [9, 10, 11, 12]]))
    assert (mask[64:n] == 0xffffffff).all()
    np.testing.assert_array_equal(mask[:64], plain_masks(list(range(-1, 63)), 2)[0])


@pytest.mark.parametrize("dtype", ["bf16", "e4m3"])
@pytest.mark.parametrize("B,hkv,g", [(300, 2, 4), (257, 1, 7), (600, 1, 2)])
@pytest.mark.parametrize("several", [False, True])
def test_single_rows_of_more_sequences_than_a_wave_plans(dtype, B, hkv, g, several):
    # no more rows than sequences: the kernel of single tokens behind the launch that plans
    rng = np.random.default_rng(B + several)
    new = np.ones(B, int)
    if several:  # some with two to four, as many of none
        order = rng.permutation(B)
        new[order[:20]], new[order[20:40]], new[order[40:100]] = 2, 4, 0
        new[order[100:120]] = 0
    assert new.sum() <= B
    lens = [int(n + x) for n, x in zip(new, np.exp(rng.uniform(0, np.log(3000), B)).astype(int) - 1)]
    for b, m in ((0, 511), (1, 512), (2, 639), (3, 640), (4, 0), (5, 1)):
        lens[b] = m
    seen = [od.masks(du.tree(rng, n))[0] if n else np.zeros((0, 0), bool) for n in new]
    for s in seen[::3]:
        s[:1] = False
    p = pu.Paged(lens, hkv, 32, dtype, seed=B)
    q = pu.bf16(rng.standard_normal((new.sum(), hkv * g, du.DH)))
    got = du.attend(p, q, new, seen, 1, junk=0xdeadbeef, pad=0)
    pu.check(got, *du.answer(p, q, new, seen))
    blind = [b for b in range(B) if len(seen[b]) and lens[b] <= new[b] and not seen[b][0].any()]
    assert blind and all((got[new[:b].sum()] == 0).all() for b in blind)

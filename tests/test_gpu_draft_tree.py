"""Masks of trees, and attention under masks of bits, against the float64 oracle."""
import numpy as np
import pytest
import torch

import draft_util as du
import paged_util as pu
from oracle import draft as od

pytestmark = pytest.mark.gpu
ce = pytest.importorskip("paper_2608_29291_amd")

JUNK = 0xdeadbeef


def run_masks(new, trees, words, base=None, rows=None):
    rows = sum(new) + 3 if rows is None else rows
    par = np.full(rows, 99, np.int32)
    flat = [p for t in trees for p in t]
    par[:len(flat)] = flat[:rows]
    d = ce.Drafts(du.up(du.offsets(new)), du.up(par))
    mask = torch.full((rows, words), 0x55555555, dtype=torch.int32, device="cuda")
    pos = torch.full((rows,), -7, dtype=torch.int32, device="cuda")
    st = torch.full((1,), -1, dtype=torch.int32, device="cuda")
    ce.ce_draft_masks(d, mask, positions=pos, base=None if base is None else du.up(np.array(base, np.int32)), status=st)
    return mask.cpu().numpy().view(np.uint32), pos.cpu().numpy(), int(st)


def check_masks(new, trees, words, base=None):
    mask, pos, st = run_masks(new, trees, words, base)
    at = 0
    for b, t in enumerate(trees):
        seen, depth = od.masks(t)
        np.testing.assert_array_equal(mask[at:at + len(t)], od.words(seen, words))
        np.testing.assert_array_equal(pos[at:at + len(t)], depth + (0 if base is None else base[b]))
        at += len(t)
    assert (mask[at:] == 0x55555555).all() and (pos[at:] == -7).all(), "rows behind the last were written"
    return st


@pytest.mark.parametrize("new,words", [([1], 1), ([0, 2, 0], 1), ([26] * 5, 1), ([33, 32, 31, 64, 65, 1, 0, 130], 5),
                                       ([300, 7], 64), ([64] * 300, 2), ([1024, 2048], 64)])
def test_masks(new, words):
    rng = np.random.default_rng(len(new))
    trees = [du.tree(rng, n) if n else [] for n in new]
    assert check_masks(new, trees, words, base=rng.integers(0, 1 << 20, len(new)).tolist()) == 0


@pytest.mark.parametrize("n", [1, 31, 32, 33, 64, 700, 2048, 9000])
def test_masks_of_chains(n):
    # with parents, and without: longer than the masks are wide, and than what a workgroup stages
    words = min(64, -(-n // 32))
    st = check_masks([n, 3], [list(range(-1, n - 1)), [-1, 0, 1]], words)
    assert st == (ce.CE_DEV_TOO_WIDE if n > 2048 else 0)
    d = ce.Drafts(du.up(du.offsets([n, 3])), rows=n + 3)
    mask = torch.zeros((n + 3, words), dtype=torch.int32, device="cuda")
    pos = torch.zeros(n + 3, dtype=torch.int32, device="cuda")
    ce.ce_draft_masks(d, mask, positions=pos)
    np.testing.assert_array_equal(mask[:n].cpu().numpy().view(np.uint32), od.words(np.tril(np.ones((n, n), bool)), words))
    np.testing.assert_array_equal(pos.cpu().numpy(), list(range(n)) + [0, 1, 2])


def test_masks_narrower_than_the_tree():
    rng = np.random.default_rng(3)
    assert check_masks([100, 20], [du.tree(rng, 100), du.tree(rng, 20)], 2) == ce.CE_DEV_TOO_WIDE


def test_masks_of_bad_trees_and_offsets():
    # parents at and behind their row, roots in the middle
    assert check_masks([6, 4], [[-1, 1, 5, 0, -3, 4], [3, 0, 0, 1000]], 1) == ce.CE_DEV_BAD_TREE
    _, _, st = run_masks([5, 9], [[-1] * 5, [-1] * 9], 1, rows=10)
    assert st & ce.CE_DEV_OVERFLOW
    d = ce.Drafts(du.up(np.array([-5, 4, 2, 1 << 30], np.int32)), du.up(np.full(8, -1, np.int32)))
    st = torch.zeros(1, dtype=torch.int32, device="cuda")
    mask = torch.zeros((8, 1), dtype=torch.int32, device="cuda")
    ce.ce_draft_masks(d, mask, status=st)
    assert int(st) & ce.CE_DEV_BAD_OFFSETS and int(st) & ce.CE_DEV_OVERFLOW


def case(new, lens, hkv, g, page, dtype, seen, words, seed=0, junk=JUNK, tol=None, **kw):
    p = pu.Paged(lens, hkv, page, dtype, seed=seed)
    rng = np.random.default_rng(seed + 1)
    q = pu.bf16(rng.standard_normal((sum(new), hkv * g, du.DH)))
    got = du.attend(p, q, new, seen, words, junk=junk, **kw)
    pu.check(got, *du.answer(p, q, new, seen))
    return p, q, got


def trees(new, seed=5):
    rng = np.random.default_rng(seed)
    return [od.masks(du.tree(rng, n))[0] if n else np.zeros((0, 0), bool) for n in new]


# few rows and many, a call of single tokens (no more rows than sequences with padding: 3 more
# rows than needed, so B is large there), trees alone, over short and over cut caches
# (many rows behind the last sequence: the call counts as a large one, and short sequences' rows
# go 128 to a tile, not 32)
PADS = [3, 12000]


@pytest.mark.parametrize("pad", PADS)
@pytest.mark.parametrize("dtype", ["bf16", "e4m3"])
@pytest.mark.parametrize("new,lens,hkv,g,page,words", [
    ([1], [1], 1, 1, 16, 1),
    ([5], [37], 2, 6, 16, 1),
    ([4, 0, 1, 3], [700, 20, 1, 3], 2, 7, 32, 1),
    ([26, 9], [1100, 2], 1, 6, 16, 2),  # nine rows of which two are in the cache
    ([64, 33, 64], [64, 1500, 90], 1, 7, 64, 2),
    ([32, 33, 1, 2], [333, 40, 2, 600], 2, 1, 256, 3),
    ([130, 70], [130, 400], 1, 4, 16, 5),
    ([2, 0, 1, 0, 0, 0, 0, 1], [900, 0, 33, 5, 0, 1, 2, 2100], 2, 4, 16, 1),
])
def test_tree_attention(dtype, new, lens, hkv, g, page, words, pad):
    case(new, lens, hkv, g, page, dtype, trees(new), words, pad=pad)


@pytest.mark.parametrize("dtype", ["bf16", "e4m3"])
@pytest.mark.parametrize("new,lens,hkv,g,words", [([26, 9], [8191, 8192], 1, 6, 1), ([40, 3, 200], [2500, 8193, 700], 1, 4, 7),
                                                  ([5, 12, 70, 1], [4000, 640, 1100, 7000], 2, 6, 3),
                                                  ([26, 40, 9], [511, 512, 600], 1, 6, 2)])
def test_small_calls_over_long_caches(dtype, new, lens, hkv, g, words):
    case(new, lens, hkv, g, 64, dtype, trees(new), words)


@pytest.mark.parametrize("pad", PADS)
@pytest.mark.parametrize("words", [2, 5])
def test_lengths_about_the_shortest_that_is_cut(words, pad):
    case([40, 33, 64, 64, 20], [639, 640, 641, 600, 64], 2, 4, 16, "bf16", trees([40, 33, 64, 64, 20]), words, pad=pad)


@pytest.mark.parametrize("pad", PADS)
@pytest.mark.parametrize("dtype", ["bf16", "e4m3"])
@pytest.mark.parametrize("new,lens,g", [([20, 45, 200], [20, 300, 517], 3), ([3, 7], [3, 2000], 2)])
def test_any_bits(dtype, new, lens, g, pad):
    # bits of any kind, behind the row itself too, and rows that see nothing at all
    rng = np.random.default_rng(11)
    seen = [rng.random((n, n)) < 0.3 for n in new]
    for s in seen:
        s[::4] = False
    _, _, got = case(new, lens, 2, g, 16, dtype, seen, 7, pad=pad)
    assert (got[0] == 0).all()  # (the first sequence has no tokens before its new ones)


# (128 rows of one query each hold more words than a tile keeps; 1500 cached keys are cut)
@pytest.mark.parametrize("dtype", ["bf16", "e4m3"])
@pytest.mark.parametrize("g,lens", [(3, [900, 150]), (1, [900, 150]), (1, [1800, 1650]), (7, [3000, 150])])
@pytest.mark.parametrize("pad", PADS)
def test_images_inside_a_prompt(dtype, g, lens, pad):
    seen = []
    for n, ends in ((300, (40, 200, 230)), (150, (1, 150))):
        s = np.tril(np.ones((n, n), bool))
        s[ends[0]:ends[1], ends[0]:ends[1]] = True
        seen.append(s)
    case([300, 150], lens, 1, g, 32, dtype, seen, 10, pad=pad)


@pytest.mark.parametrize("B", [1, 70, 300])
def test_batches_whose_chunks_are_rounded_up(B):
    # lengths about one and a half shares: counts rounded up may be more than the places, and are not then
    new = [40] * B if B < 300 else [9 + b % 3 for b in range(B)]
    lens = [1100 + 7 * (b % 50) for b in range(B)] if B > 1 else [9000]
    p = pu.Paged(lens, 2, 64, "bf16", k=[np.zeros((m, 2, du.DH), np.float32) for m in lens],
                 v=[pu.bf16(np.full((m, 2, du.DH), 1.0) + np.arange(m)[:, None, None] % 3) for m in lens])
    q = np.ones((sum(new), 14, du.DH), np.float32)
    seen = trees(new)
    got = du.attend(p, q, new, seen, 2)
    # all scores are 0, so every output is the mean of the values seen: 1 + (0 + 1 + 2 of the keys) / their number
    at = 0
    for b, n in enumerate(new):
        vis = du.visible(seen[b], n, lens[b])
        want = (vis * (1 + np.arange(lens[b]) % 3)).sum(1) / vis.sum(1)
        # weights of 1 are exact; the output's rounding is half a step, and so that of a float32 sum and quotient
        assert np.abs(got[at:at + n] - want[:, None, None]).max() <= 2 * 2.0 ** -8 + 2.0 ** -10
        at += n


@pytest.mark.parametrize("pad", PADS)
def test_masks_narrower_than_the_new_tokens(pad):
    seen = [np.ones((70, 70), bool)]
    p = pu.Paged([100], 1, 16, "bf16")
    q = pu.bf16(np.random.default_rng(0).standard_normal((70, 2, du.DH)))
    got = du.attend(p, q, [70], seen, 2, pad=pad)
    seen[0][:, 64:] = False  # token 64 on has no bit
    pu.check(got, *du.answer(p, q, [70], seen))


@pytest.mark.parametrize("dtype", ["bf16", "e4m3"])
@pytest.mark.parametrize("n,pad", [(5, 3), (60, 3), (60, 12000)])
def test_what_is_hidden_has_no_influence(dtype, n, pad):
    """NaN, infinities and huge values in keys and values that no row, or not every row sees."""
    rng = np.random.default_rng(2)
    seen = od.masks(du.tree(rng, n))[0]
    m = 200 + n
    k, v = (pu.bf16(rng.standard_normal((m, 1, du.DH))) for _ in range(2))
    bad = 200 + np.array([n - 1, n // 2])
    k[bad[0]], v[bad[0]] = np.nan, np.nan
    v[bad[1]] = np.nan if dtype == "e4m3" else np.inf
    p = pu.Paged([m], 1, 16, dtype, k=[k], v=[v])
    q = pu.bf16(rng.standard_normal((n, 4, du.DH)))
    got = du.attend(p, q, [n], [seen], 2, junk=JUNK, pad=pad)
    want, top = du.answer(p, q, [n], [seen])
    with np.errstate(invalid="ignore"):
        inf = np.isinf(want)
        np.testing.assert_array_equal(np.isinf(got), inf)
        pu.check(np.where(inf, 0, got), np.where(inf, 0, want), top)
    assert np.isfinite(got[0]).all()


@pytest.mark.parametrize("n,pad", [(3, 3), (40, 3), (40, 12000)])
def test_a_row_that_sees_scores_of_minus_infinity_only(n, pad):
    k = np.ones((n, 1, du.DH), np.float32)
    k[0] = -np.inf
    p = pu.Paged([n], 1, 16, "bf16", k=[k])
    q = np.ones((n, 2, du.DH), np.float32)
    seen = np.eye(n, dtype=bool)
    seen[1] = False
    got = du.attend(p, q, [n], [seen], 2, pad=pad)
    assert np.isnan(got[0]).all() and (got[1] == 0).all() and np.isfinite(got[2:]).all()


def test_a_chain_is_causal_attention():
    p = pu.Paged([500, 77, 4000], 2, 16, "bf16")
    new = [9, 40, 100]
    q = pu.bf16(np.random.default_rng(9).standard_normal((sum(new), 6, du.DH)))
    seen = [np.tril(np.ones((n, n), bool)) for n in new]
    got = du.attend(p, q, new, seen, 4)
    want = pu.attend(p, q, new, True)
    assert np.abs(got - want).max() <= 2 * pu.TOL * 5


@pytest.mark.parametrize("new", [[64, 20, 33], [2, 3, 1]])
def test_repeats_streams_and_scratch(new):
    p = pu.Paged([5000, 41, 1033], 2, 32, "e4m3")
    q = pu.bf16(np.random.default_rng(9).standard_normal((sum(new), 8, du.DH)))
    seen = trees(new)
    first = du.attend(p, q, new, seen, 2)
    for kw in ({}, {"ws": False}, {"stream": torch.cuda.Stream()}, {"ws": False, "stream": torch.cuda.Stream()}):
        np.testing.assert_array_equal(du.attend(p, q, new, seen, 2, **kw), first)


def test_spaced_queries_and_a_call_of_single_rows():
    # rows of a fused projection; 40 sequences of a row each, and no padding: the kernel of single tokens
    B = 40
    lens = [1 + 37 * b for b in range(B)]
    p = pu.Paged(lens, 2, 16, "bf16")
    rng = np.random.default_rng(1)
    q = pu.bf16(rng.standard_normal((B, 8, du.DH)))
    qd = torch.zeros((B, 13, du.DH), dtype=torch.bfloat16, device="cuda")
    qd[:, 2:10] = du.up(q).to(torch.bfloat16)
    bits = np.arange(B) % 3 != 0
    seen = [np.array([[x]]) for x in bits]
    o = torch.empty((B, 8, du.DH), dtype=torch.bfloat16, device="cuda")
    ce.ce_paged_tree_attention(p.cache(), qd[:, 2:10], o, du.up(du.offsets([1] * B)), du.up(np.array(lens, np.int32)),
                               du.device_mask(seen, 1, B, JUNK), du.DH ** -0.5)
    pu.check(o.float().cpu().numpy(), *du.answer(p, q, [1] * B, seen))


def test_mask_rows_of_another_tensor_are_refused():
    p = pu.Paged([50], 1, 16, "bf16")
    q = torch.zeros((4, 2, du.DH), dtype=torch.bfloat16, device="cuda")
    off, lens = du.up(du.offsets([4])), du.up(np.array([50], np.int32))
    for mask in (torch.zeros((3, 1), dtype=torch.int32).cuda(), torch.zeros((4, 1), dtype=torch.int64).cuda(),
                 torch.zeros(4, dtype=torch.int32).cuda(), torch.zeros((4, 2), dtype=torch.int32).cuda()[:, :1],
                 torch.zeros((4, 1), dtype=torch.int32), None):
        with pytest.raises(ValueError):
            ce.ce_paged_tree_attention(p.cache(), q, q.clone(), off, lens, mask, 0.1)

"""Values at the ends of their range in attention over the paged cache: infinite scores beside
finite rows, scores so large that one key has all the weight,
softmax scales times key scales that leave float32, value scales next to zero."""
import numpy as np
import pytest

import paged_util as U

pytestmark = pytest.mark.gpu

SHAPES = [([1, 1], [900, 40]), ([3, 2], [900, 40]), ([150, 40], [1500, 64])]  # single tokens, few rows, tiles


def rows(n, heads, seed=1):
    return U.bf16(np.random.default_rng(seed).standard_normal((n, heads, U.DH)))


def go(p, q, new, scale=U.DH ** -0.5):
    """Outputs of rows q, causal."""
    import torch
    import paper_2608_29291_amd as ce
    qd = torch.from_numpy(q).to(torch.bfloat16).cuda()
    o = torch.full_like(qd, 77.0)
    i32 = lambda x: torch.tensor(x, dtype=torch.int32).cuda()
    ce.ce_paged_attention(p.cache(), qd, o, i32([0] + np.cumsum(new).tolist()), i32(p.lens), True, scale)
    return o.float().cpu().numpy()


@pytest.mark.parametrize("new,lens", SHAPES[1:])
def test_infinite_scores_touch_the_rows_that_see_them(new, lens):
    """Keys of -infinity weigh nothing, a whole chunk of them too. A key of +infinity near the
    end makes NaN of the rows that see it; earlier rows, other heads and the next sequence
    stay finite."""
    p = U.Paged(lens, 2, 16, "bf16", seed=21)
    k = [x.copy() for x in p.k]
    k[0][:700, 0, 0] = -np.inf
    k[0][lens[0] - new[0] + new[0] // 2, 1, 0] = np.inf
    p = U.Paged(lens, 2, 16, "bf16", seed=21, k=k)
    q = rows(sum(new), 12)
    q[:, :, 0] = np.abs(q[:, :, 0]) + 0.5
    q[0, 1, 0] = -1.0  # +infinity from the first key on
    want, top = p.answer(q, new, True, U.DH ** -0.5)
    bad = np.isnan(want).all(2)
    for r in range(sum(new)):
        assert bad[r].tolist() == [(h == 1 and r == 0) or (h >= 6 and new[0] // 2 <= r < new[0]) for h in range(12)]
    U.check(go(p, q, new), want, top)


def by_far(p, q, new, least=2.0 ** -12):
    """Rows and heads whose highest score is ahead of all others by `least` of its size: far more
    than a fp32 sum of 128 products errs by (about 2^-16 of it)."""
    at, sure = 0, np.zeros(q.shape[:2], bool)
    g = q.shape[1] // p.hkv
    for b, n in enumerate(new):
        for i in range(n):
            for h in range(q.shape[1]):
                s = np.sort(np.float64(p.k_used[b][:p.lens[b] - n + i + 1, h // g]) @ np.float64(q[at + i, h]))
                sure[at + i, h] = len(s) < 2 or s[-1] - s[-2] > least * np.abs(s).max()
        at += n
    return sure


@pytest.mark.parametrize("new,lens", SHAPES)
@pytest.mark.parametrize("size,scale", [(2e3, 0.1), (3e4, 0.1), (1e6, 0.1), (1e9, 0.1), (1e18, 100.0)])
def test_scores_of_any_size(size, scale, new, lens):
    """From 1e6 to past float32's range: the output is the highest key's value."""
    rng = np.random.default_rng(25)
    k = [U.bf16(rng.standard_normal((n, 2, U.DH)) * size) for n in lens]
    p = U.Paged(lens, 2, 16, "bf16", seed=25, k=k)
    q = U.bf16(rows(sum(new), 12) * size)
    want, top = p.answer(q, new, True, float(np.float32(scale)))
    sure = by_far(p, q, new)
    assert sure.mean() > 0.98
    got = go(p, q, new, scale)
    assert np.isfinite(got).all()
    assert (np.abs(got - want)[sure] <= U.TOL * top[sure][:, None]).all()


@pytest.mark.parametrize("new,lens", SHAPES[1:])
def test_unseen_values_beside_large_scores(new, lens):
    """A NaN value behind a row's mask: that output is formed again, by the same exponents."""
    rng = np.random.default_rng(26)
    k = [U.bf16(rng.standard_normal((n, 2, U.DH)) * 1e6) for n in lens]
    v = [U.bf16(rng.standard_normal((n, 2, U.DH))) for n in lens]
    v[0][-1, :, 5] = np.nan
    p = U.Paged(lens, 2, 16, "bf16", seed=26, k=k, v=v)
    q = U.bf16(rows(sum(new), 12) * 1e6)
    want, top = p.answer(q, new, True, float(np.float32(0.1)))
    sure = by_far(p, q, new)
    assert sure.mean() > 0.98 and np.isnan(want[new[0] - 1, :, 5]).all() and np.isnan(want).sum() == 12
    got = go(p, q, new, 0.1)
    U.check(got[sure][:, None], want[sure][:, None], top[sure][:, None])


@pytest.mark.parametrize("new,lens", SHAPES[1:])
def test_unseen_values_beside_a_page_that_is_none(new, lens):
    """An output that is formed again counts the keys of a missing page, all zeros, as well."""
    v = [U.bf16(np.random.default_rng(27).standard_normal((n, 2, U.DH))) for n in lens]
    v[0][-1, :, 5] = np.nan
    for dtype in ("bf16", "e4m3"):
        p = U.Paged(lens, 2, 16, dtype, seed=27, v=v)
        for b, col in ((0, 3), (0, 40), (1, 0)):
            p.table[b, col] = -1
            for x in (p.k_used[b], p.v_used[b]):
                x[16 * col:16 * col + 16] = 0.0
        q = rows(sum(new), 12)
        U.check(go(p, q, new), *p.answer(q, new, True, U.DH ** -0.5))


def quantized(lens, ks, vs, seed=22):
    """8-bit pages of standard normal values under given scales."""
    p = U.Paged(lens, 2, 16, "e4m3", seed=seed, scales=False)
    p.ks, p.vs = np.full(2, ks, np.float32), np.full(2, vs, np.float32)
    p.k_used = [x * np.float64(p.ks[0]) for x in p.k_used]
    p.v_used = [x * np.float64(p.vs[0]) for x in p.v_used]
    return p


@pytest.mark.parametrize("new,lens", SHAPES)
@pytest.mark.parametrize("scale,ks", [(1e-10, 1e-36), (1e-30, 1e-30), (1e-44, 0.02), (1e-3, 1e-40)])
def test_scores_near_zero(scale, ks, new, lens):
    """softmax scale times key scale rounds to zero or next to it: every key that is seen has
    the same weight, to within 2^-20."""
    p = quantized(lens, ks, 1.0)
    q = rows(sum(new), 12)
    U.check(go(p, q, new, scale), *p.answer(q, new, True, float(np.float32(scale))))


def test_a_denormal_softmax_scale():
    p = U.Paged([900, 40], 2, 16, "bf16", seed=23)
    for new in ([1, 1], [3, 2], [80, 40]):
        q = rows(sum(new), 12)
        U.check(go(p, q, new, 1e-44), *p.answer(q, new, True, float(np.float32(1e-44))))


@pytest.mark.parametrize("new,lens", SHAPES)
def test_a_score_scale_past_float32(new, lens):
    """The two scales multiply to 1e40 and the queries are that small: the scores are ordinary
    float32 numbers (near 1e11), so far apart that the highest takes all the weight."""
    p = quantized(lens, 1e10, 1.0)
    q = U.bf16(rows(sum(new), 12) * 1e-30)
    want, top = p.answer(q, new, True, float(np.float32(1e30)))
    sure = by_far(p, q, new)
    assert sure.mean() > 0.99
    got = go(p, q, new, 1e30)
    assert np.isfinite(got).all()
    err = np.abs(got - want)[sure]
    assert (err <= U.TOL * top[sure][:, None]).all()


@pytest.mark.parametrize("vs", [1.25e-38, 1e-36, 1e30])
def test_value_scales_far_from_one(vs):
    """Many keys of one weight: the quotient vs / (sum of weights) would be a float32 with a few
    bits left, the output is an ordinary one."""
    keys, times = 4096, 150
    p = U.Paged([keys], 1, 256, "e4m3", seed=24, scales=False, v=[np.full((keys, 1, U.DH), 448.0)])
    n = keys // 256
    p.table = np.tile(p.table[:, :n], (1, times))
    p.lens = [keys * times]
    p.ks, p.vs = np.ones(1, np.float32), np.full(1, vs, np.float32)
    want = 448.0 * np.float64(p.vs[0])
    for new in ([1], [2], [40]):
        got = go(p, np.zeros((sum(new), 2, U.DH), np.float32), new)
        assert (np.abs(got - want) <= U.TOL * want).all(), (new, got.min(), got.max(), want)

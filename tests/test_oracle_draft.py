"""The oracle of drafted decoding against its definitions (CPU)."""
import itertools

import numpy as np
import pytest

from oracle import draft as od
from oracle import paged as op


def test_masks_by_hand():
    seen, depth = od.masks([-1, 0, 0, 1, 3, 2])
    assert depth.tolist() == [0, 1, 1, 2, 3, 2]
    assert [np.flatnonzero(r).tolist() for r in seen] == [[0], [0, 1], [0, 2], [0, 1, 3], [0, 1, 3, 4], [0, 2, 5]]
    assert od.words(seen, 1).ravel().tolist() == [1, 3, 5, 11, 27, 37]
    seen, _ = od.masks([-1, 5, 1])  # a parent behind its row is none
    assert [np.flatnonzero(r).tolist() for r in seen] == [[0], [1], [1, 2]]


def test_chain_masks_are_causal_attention():
    rng = np.random.default_rng(0)
    q, k, v = rng.standard_normal((5, 4, 8)), rng.standard_normal((9, 2, 8)), rng.standard_normal((9, 2, 8))
    seen = np.concatenate([np.ones((5, 4), bool), od.masks([-1, 0, 1, 2, 3])[0]], 1)
    np.testing.assert_array_equal(od.attend(q, k, v, seen, 0.3), op.attend(q, k, v, True, 0.3))


def test_sample_is_the_inverse_of_the_running_sum():
    w = np.array([0.0, 1.0, 0.0, 2.0, 1.0, 0.0])
    assert [od.sample(w, u) for u in (0.0, 0.24, 0.25, 0.7, 0.75, 0.999, 1.0)] == [1, 1, 3, 3, 4, 4, 4]


def _first_tokens(p, q, children, n):
    """Exact distribution of the first token after row 0, over grids of n numbers whose cells no
    border crosses."""
    V = len(p)
    got = np.zeros(V)
    grid = (np.arange(n) + 0.5) / n
    logits = np.log(np.where(p > 0, p, 1e-300))[None].repeat(children + 1, 0)
    for xs in itertools.product(range(V), repeat=children):
        chance = np.prod([q[x] for x in xs])
        if chance == 0:
            continue
        for us in itertools.product(grid, repeat=children + 1):
            walk, nxt = od.verify([-1] + [0] * children, [0] + list(xs), logits, 1.0, [us[-1]] * (children + 1),
                                  q[None].repeat(children + 1, 0), [0.0] + list(us[:-1]))
            got[xs[walk[1] - 1] if len(walk) > 1 else nxt] += chance / n ** (children + 1)
    return got


@pytest.mark.parametrize("children", [1, 2])
def test_drawn_drafts_keep_the_targets_distribution(children):
    # acceptance at 1/2 and 1, residuals on the first token only: all borders are multiples of 1/4
    p, q = np.array([0.5, 0.25, 0.25]), np.array([0.25, 0.5, 0.25])
    np.testing.assert_allclose(_first_tokens(p, q, children, 4), p, atol=1e-12)


def test_chosen_drafts_keep_the_targets_distribution():
    p = np.array([0.5, 0.125, 0.375])
    got = np.zeros(3)
    for u in (np.arange(8) + 0.5) / 8:
        walk, nxt = od.verify([-1, 0, 0], [0, 2, 1], np.log(p)[None].repeat(3, 0), 1.0, [u] * 3)
        got[[0, 2, 1][walk[1]] if len(walk) > 1 else nxt] += 1 / 8
    np.testing.assert_allclose(got, p, atol=1e-12)


def test_verify_special_rows():
    inf, nan = np.inf, np.nan
    one = lambda row, t=1.0, u=0.5: od.verify([-1], [0], np.array([row]), t, [u])
    assert one([nan, -inf]) == ([0], -1)
    assert one([0.0, inf, -inf, inf], u=0.6) == ([0], 3)
    assert one([1.0, 3.0, 3.0, nan], t=0.0) == ([0], 1)
    assert one([1.0, 3.0, 3.0], t=nan) == ([0], 1)
    assert od.verify(None, [], np.zeros((0, 3)), 1.0, []) == ([], -1)


def test_keep_by_hand():
    assert od.keep(list("abcdef"), 2, [0, 2, 3]) == list("abceff")
    assert od.keep(list("abcdef"), 2, [0, 2, 2]) == list("abceef")
    assert od.keep(list("abcdef"), 2, [1, 4]) == list("abddef")


def test_rotary_by_hand():
    x = np.array([[[1.0, 2.0, 3.0, 4.0, 5.0]]])
    f, pos = [np.pi / 2, np.pi / 4], np.array([[1], [4]])
    np.testing.assert_allclose(od.rotary(x, pos, f, [0, 1], False)[0, 0], [-3, -2, 1, -4, 5], atol=1e-12)
    np.testing.assert_allclose(od.rotary(x, pos, f, [0, 1], True)[0, 0], [-2, 1, -3, -4, 5], atol=1e-12)
    np.testing.assert_array_equal(od.rotary(x, pos, f, [0, 1], True, index=[7]), x)

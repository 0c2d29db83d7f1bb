"""Pins of the paged cache's oracle: a worked reservation, invariants of a long
random run, the 8-bit format against torch's, attention against the packed oracle."""
import numpy as np
import pytest

import oracle
from oracle import paged as op


def test_reserve_by_hand():
    # pages of 4; sequence 0 holds 5 tokens (pages 7, 3), 1 holds 4 (page 0), 2 none
    table = np.array([[7, 3, -1, -1], [0, -1, -1, -1], [-1, -1, -1, -1]])
    lens, start, slots, t, free, why = op.reserve([5, 4, 0], [4, 1, 2], 4, table, [9, 8, 6, 5, 2])
    assert lens == [9, 5, 2] and start == [5, 4, 0] and why == ["", "", ""]
    assert t[0].tolist() == [7, 3, 2, -1] and t[1].tolist() == [0, 5, -1, -1] and t[2].tolist() == [6, -1, -1, -1]
    assert slots == [13, 14, 15, 8, 20, 24, 25]
    assert free == [9, 8]
    # 0 is handed on: its pages go back in table order, the last on top
    lens, start, slots, t, free, why = op.reserve([5, 4, 0], [1, 0, 0], 4, table, [9], reset=[1, 0, 0])
    assert lens == [1, 4, 0] and t[0].tolist() == [3, 3, -1, -1] and free == [9, 7] and slots == [12]


def test_reserve_refusals_by_hand():
    table = np.full((4, 2), -1)
    # 1 wants two pages of the one left, 2 one: refused behind it; 3 needs none
    lens, start, slots, _, free, why = op.reserve([0, 0, 0, 0], [4, 8, 1, 0], 4, table, [5, 6])
    assert why == ["", "pages", "pages", ""] and start == [0, -1, -1, 0] and lens == [4, 0, 0, 0]
    assert slots == [24, 25, 26, 27] + [-1] * 9 and free == [5]
    # too long for its two pages: refused, and the pages stay for others
    lens, _, _, _, free, why = op.reserve([0, 0, 0, 0], [9, 8, 0, 0], 4, table, [5, 6])
    assert why == ["long", "", "", ""] and lens == [0, 8, 0, 0] and free == []


def test_reserve_keeps_every_page_once():
    rng = np.random.default_rng(0)
    B, page, n = 9, 4, 60
    lens, table, free = [0] * B, np.full((B, 12), -1), list(rng.permutation(n))
    for _ in range(200):
        new, reset = rng.integers(0, 9, B), rng.random(B) < 0.15
        lens, start, slots, table, free, why = op.reserve(lens, new, page, table, free, reset)
        held = [int(table[b, j]) for b in range(B) for j in range(-(-lens[b] // page))]
        assert sorted(held + free) == list(range(n))
        at = 0
        for b in range(B):
            for i in range(new[b]):
                t = start[b] + i
                assert slots[at] == (-1 if why[b] else table[b, t // page] * page + t % page)
                at += 1


def test_e4m3_against_torch():
    torch = pytest.importorskip("torch")
    x = torch.cat([torch.arange(65536, dtype=torch.int32).to(torch.int16).view(torch.bfloat16).float(),
                   torch.randn(20000) * 100, torch.linspace(-0.02, 0.02, 4001)])
    x = x[~torch.isnan(x)]
    want = x.clamp(-448, 448).to(torch.float8_e4m3fn)
    np.testing.assert_array_equal(op.e4m3(x.numpy()), want.view(torch.uint8).numpy())
    codes = np.arange(256, dtype=np.uint8)
    np.testing.assert_array_equal(op.e4m3_value(codes), torch.from_numpy(codes).view(torch.float8_e4m3fn).double().numpy())
    assert op.e4m3([np.nan, np.inf, -np.inf]).tolist() == [0x7f, 0x7e, 0xfe]


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("n_q,n_k", [(1, 7), (5, 5), (4, 9), (6, 2), (3, 0)])
def test_attend_is_the_packed_attention(n_q, n_k, causal):
    rng = np.random.default_rng(n_q * 10 + n_k)
    q, k, v = rng.standard_normal((n_q, 6, 16)), rng.standard_normal((n_k, 2, 16)), rng.standard_normal((n_k, 2, 16))
    want = oracle.attention.attention(q, k, v, [0, n_q], [0, n_k], 2, causal, 0.3)
    np.testing.assert_allclose(op.attend(q, k, v, causal, 0.3), want, atol=1e-13)


def test_attend_ignores_what_is_not_seen():
    rng = np.random.default_rng(4)
    q, k, v = (rng.standard_normal((5, 1, 8)) for _ in range(3))
    want = op.attend(q, k, v, True, 1.0)
    k[4], v[3] = np.nan, np.inf
    got = op.attend(q, k, v, True, 1.0)
    np.testing.assert_array_equal(got[:3], want[:3])
    assert np.isinf(got[3]).all() and np.isnan(got[4]).all()
    k[:] = -np.inf
    assert np.isnan(op.attend(np.abs(q), k, v, True, 1.0)).all()  # 0 / 0

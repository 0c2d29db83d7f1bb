"""Rotary positions against the float64 oracle."""
import numpy as np
import pytest
import torch

import draft_util as du
from oracle import draft as od

pytestmark = pytest.mark.gpu
ce = pytest.importorskip("paper_2608_29291_amd")

# A turn is off by 2^-28, 2.4e-8 rad, and once more by the angle's rounding to float32 (half a step of at
# most pi / 4, 3e-8); cosine and sine are polynomials of four and five steps, each rounded to a size of at
# most 1 (the last two count, 2^-24 each, the others a quarter and less: 3 2^-24), so 2.4e-8 + 3e-8 + 1.8e-7
# on a value below 1; the two products and their sum add 2 2^-24 of |x1| + |x2|. Together below 6 2^-24
# of |x1| + |x2|, and the output's own rounding.
ANGLE = 6 * 2.0 ** -24


def check(y, want, x, pairs, interleaved, dtype):
    x = np.abs(np.array(x, np.float64))
    first, second = (slice(0, 2 * pairs, 2), slice(1, 2 * pairs, 2)) if interleaved else (slice(0, pairs), slice(pairs, 2 * pairs))
    lim = np.zeros(x.shape)
    lim[..., first] = lim[..., second] = ANGLE * (x[..., first] + x[..., second])
    # (half a step of the output, of what the sum was before it)
    lim = lim + torch.finfo(dtype).eps / 2 * (np.abs(want) + lim)
    lim[..., 2 * pairs:] = 0
    err = np.abs(y - want)
    assert (err <= lim).all(), (err / np.maximum(lim, 1e-30)).max()


def make(rows, heads, dim, dtype, seed=0):
    g = np.random.default_rng(seed)
    return torch.from_numpy(g.standard_normal((rows, heads, dim)).astype(np.float32)).to(dtype)


def axes_of(pairs, n):
    return [i * n // pairs for i in range(pairs)]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("rows,heads,dim,pairs,axes", [
    (1, 1, 128, 64, 1), (5, 3, 128, 32, 3), (7, 4, 64, 32, 2), (3, 2, 80, 40, 3), (4, 5, 72, 36, 4), (9, 4, 96, 20, 1),
    (2, 4, 256, 128, 2), (6, 4, 48, 5, 2), (3, 8, 254, 1, 1), (300, 9, 128, 64, 3), (3000, 30, 64, 16, 1), (3000, 30, 128, 64, 3), (2, 4, 2, 1, 1)])
def test_turn(dtype, interleaved, rows, heads, dim, pairs, axes):
    x = make(rows, heads, dim, dtype)
    rng = np.random.default_rng(1)
    pos = rng.integers(0, 40000, (axes, rows)).astype(np.int32)
    freqs, of = ce.rotary_freqs(2 * pairs), axes_of(pairs, axes)
    r = ce.Rotary(freqs, of, interleaved=interleaved)
    y = torch.full_like(x, 9.0).cuda()
    ce.ce_rotary(r, x.cuda(), y, du.up(pos))
    some = np.unique(np.concatenate([np.arange(min(rows, 40)), [rows - 1]]))
    xs = x[some].double().numpy()
    want = od.rotary(xs, pos[:, some], freqs, of, interleaved)
    check(y[some].double().cpu().numpy(), want, xs, pairs, interleaved, dtype)
    # in place, of rows of a fused projection
    fused = torch.zeros((rows, heads + 4, dim), dtype=dtype, device="cuda")
    if (heads + 4) * dim % 8 == 0 and 2 * dim * fused.element_size() % 16 == 0:
        part = fused[:, 2:2 + heads]
        part.copy_(x)
        ce.ce_rotary(r, part, part, du.up(pos))
        assert torch.equal(part, y)
        assert (fused[:, :2] == 0).all() and (fused[:, 2 + heads:] == 0).all()


@pytest.mark.parametrize("interleaved", [False, True])
def test_packed_rows_keep_their_tokens_positions(interleaved):
    n, rows = 500, 200
    rng = np.random.default_rng(4)
    index = np.sort(rng.permutation(n)[:rows]).astype(np.int32)
    index[[3, 50, 199]] = [-1, n, 1 << 30]  # no token's: the row is not turned
    pos = rng.integers(0, 5000, (3, n)).astype(np.int32)
    x = make(rows, 3, 128, torch.float32)
    freqs, of = ce.rotary_freqs(64), axes_of(32, 3)
    r = ce.Rotary(freqs, of, interleaved=interleaved)
    y = torch.zeros_like(x).cuda()
    ce.ce_rotary(r, x.cuda(), y, du.up(pos), index=du.up(index))
    want = od.rotary(x.numpy(), pos, freqs, of, interleaved, index=index)
    check(y.double().cpu().numpy(), want, x.numpy(), 32, interleaved, torch.float32)
    assert torch.equal(y[[3, 50, 199]].cpu(), x[[3, 50, 199]])
    z = x.cuda()
    ce.ce_rotary(r, z, z, du.up(pos), index=du.up(index))
    assert torch.equal(z, y)


def test_far_and_negative_positions():
    pos = np.array([[0, 1, -1, 2 ** 31 - 1, -2 ** 31, 123456789, -987654321, 2 ** 30]], np.int32)
    x = make(8, 2, 64, torch.float32)
    freqs = [1.0, 0.9999, 3.0, 64.0, -1.0, -0.3, 1e-9, 2.0 ** -31, np.pi, np.pi / 2, np.pi / 4, 3 * np.pi / 4] + \
        ce.rotary_freqs(40, 5e5)
    r = ce.Rotary(freqs)
    y = torch.zeros_like(x).cuda()
    ce.ce_rotary(r, x.cuda(), y, du.up(pos))
    check(y.double().cpu().numpy(), od.rotary(x.numpy(), pos, freqs, [0] * 32, False), x.numpy(), 32, False, torch.float32)


@pytest.mark.parametrize("interleaved", [False, True])
def test_inverse_undoes_the_turn_and_is_its_gradient(interleaved):
    x, g = make(50, 4, 96, torch.float32), make(50, 4, 96, torch.float32, seed=7)
    pos = du.up(np.random.default_rng(3).integers(-3000, 3000, (2, 50)).astype(np.int32))
    r = ce.Rotary(ce.rotary_freqs(64), axes_of(32, 2), interleaved=interleaved)
    xd, gd = x.cuda(), g.cuda()
    y, back, dx = torch.empty_like(xd), torch.empty_like(xd), torch.empty_like(xd)
    ce.ce_rotary(r, xd, y, pos)
    ce.ce_rotary(r, y, back, pos, inverse=True)
    ce.ce_rotary(r, gd, dx, pos, inverse=True)
    # two turns, each off by ANGLE and half a step of a sum of at most |x1| + |x2| < 2 * 1.5 max |x|
    assert (back - xd).abs().max() <= 2 * (ANGLE + 2.0 ** -24) * 2 * 1.5 * x.abs().max()
    # the formula's gradient: the oracle's turn back
    want = od.rotary(g.numpy(), pos.cpu().numpy(), ce.rotary_freqs(64), axes_of(32, 2), interleaved, inverse=True)
    check(dx.double().cpu().numpy(), want, g.numpy(), 32, interleaved, torch.float32)
    # and differences: the turn is linear, so <g, turn(x + h) - turn(x)> = <dx, h>
    h = make(50, 4, 96, torch.float32, seed=9).cuda()
    y2 = torch.empty_like(xd)
    ce.ce_rotary(r, xd + h, y2, pos)
    lhs = ((y2.double() - y.double()) * gd.double()).sum()
    rhs = (dx.double() * h.double()).sum()
    # each of the 50 4 96 terms is off by 4 (ANGLE + 2^-24) (|x1| + |x2|) |g| at most, with values below 5
    assert (lhs - rhs).abs() <= 50 * 4 * 96 * 4 * (ANGLE + 2.0 ** -24) * 10 * 5


def test_special_values_and_empty_calls():
    x = make(3, 1, 32, torch.float32)
    x[1, 0, 3] = float("inf")
    x[2, 0, 20] = float("nan")
    y = torch.zeros_like(x).cuda()
    pos = du.up(np.array([5, 6, 7], np.int32))
    ce.ce_rotary(ce.Rotary(ce.rotary_freqs(16)), x.cuda(), y, pos)
    bad = ~torch.isfinite(y.cpu())
    assert set(map(tuple, bad.nonzero().tolist())) == {(1, 0, 3), (1, 0, 11), (2, 0, 20)}
    e = torch.zeros((0, 4, 32), device="cuda")
    ce.ce_rotary(ce.Rotary([1.0]), e, e, pos)
    z = torch.zeros((2, 4, 32), device="cuda")
    with pytest.raises(ValueError):
        ce.ce_rotary(ce.Rotary([1.0, 1.0], [0, 1]), z, z, pos)  # one axis of positions
    with pytest.raises(ce.CERouterError):
        ce.ce_rotary(ce.Rotary([1.0] * 17), z, z, pos)  # more pairs than a head has
    with pytest.raises(ValueError):
        ce.ce_rotary(ce.Rotary([1.0]), z.half(), z.half(), pos)
    # without positions no row is turned
    w = torch.zeros_like(x).cuda()
    ce.ce_rotary(ce.Rotary([1.0]), x.cuda(), w, torch.zeros(0, dtype=torch.int32, device="cuda"))
    assert torch.equal(w.cpu().nan_to_num(), x.nan_to_num())

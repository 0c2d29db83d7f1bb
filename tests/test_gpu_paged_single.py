"""The kernel of single tokens (no more rows of q than sequences, at most eight heads a
key/value head) where it differs from the one of many rows: how many chunks a cut
sequence has and in how many levels they meet, what a masked, missing or infinite value
may touch, calls in flight on two streams. Every call here is checked to have taken
that kernel: by its workspace, and the cut ones by the partial results it left there.
"""
import numpy as np
import pytest

import paged_util as U

pytestmark = pytest.mark.gpu

PLACES = 512
COUNTERS = 3 * PLACES * 8   # bytes in front of the partial results, up to 256 sequences
SLOT = 32 * (U.DH + 2)      # floats of a partial result: outputs, maxima, sums of 32 rows
BYTES = COUNTERS + PLACES * SLOT * 4


def rows(n, heads, seed=1, spread=1.0):
    return U.bf16(np.random.default_rng(seed).standard_normal((n, heads, U.DH)) * spread)


def i32(x):
    import torch
    return torch.tensor(x, dtype=torch.int32).cuda()


def single(p, q, new=None, causal=True, scale=U.DH ** -0.5, pad=0):
    """Outputs of rows q (behind them `pad` more that belong to no sequence) and the
    partial results that the call left."""
    import torch
    import paper_2608_29291_amd as ce
    B = len(p.lens)
    new = [1] * B if new is None else new
    c = p.cache()
    qd = torch.full((len(q) + pad, *q.shape[1:]), float("nan"), dtype=torch.bfloat16, device="cuda")
    qd[:len(q)] = torch.from_numpy(q).to(torch.bfloat16).cuda()
    o = torch.full_like(qd, 77.0)
    assert sum(new) == len(q) and len(qd) <= B <= 256
    need = ce.ce_paged_workspace_size(c, len(qd), q.shape[1])
    assert need == (BYTES if p.width * p.page >= 512 else 0)
    ws = torch.full((max(need, 256),), 0xff, dtype=torch.uint8, device="cuda")  # NaN
    off = i32([0] + np.cumsum(new).tolist())
    ce.ce_paged_attention(c, qd, o, off, i32(p.lens), causal, scale, ws=ws)
    torch.cuda.synchronize()
    assert (o[len(q):] == 77.0).all(), "rows behind the last were written"
    top = ws[COUNTERS:].view(torch.float32).view(PLACES, SLOT)[:, 32 * U.DH] if need else torch.empty(0)
    return o[:len(q)].float().cpu().numpy(), int((~torch.isnan(top)).sum())


def long_cache(lens, heads_kv, page, dtype, seed):
    """Sequences over the same 8192 keys again and again."""
    keys = 8192
    p = U.Paged([keys], heads_kv, page, dtype, seed=seed)
    n = keys // page
    times = -(-max(lens) // keys)
    p.table = np.repeat(np.concatenate([np.tile(p.table[:, :n], (1, times)), p.table[:, n:]], 1), len(lens), 0)
    p.width, p.lens = p.table.shape[1], list(lens)
    k, v = p.k_used[0], p.v_used[0]
    kv = {m: [np.resize(x, (m, *x.shape[1:])) for x in (k, v)] for m in set(lens)}
    p.k_used, p.v_used = [kv[m][0] for m in lens], [kv[m][1] for m in lens]
    return p


# lengths, heads and the chunks that a sequence and key/value head alone is cut into. 128
# keys is the least chunk, so 128 n keys of one unit are n chunks, up to half of the places.
LEVELS = {
    "none": ([639], 7, 0),
    "one": ([128 * 10], 7, 10),
    "one_full": ([8192], 7, 16),               # more chunks are made 16 up to 512 keys each
    "two_rest_of_one": ([128 * 65], 7, 65),    # 16, 16, 16, 16 and 1
    "two_rest": ([128 * 78], 8, 78),           # and 14
    "two_full": ([128 * 80], 1, 80),
}


@pytest.mark.parametrize("dtype", ["bf16", "e4m3"])
@pytest.mark.parametrize("name", LEVELS)
def test_levels(name, dtype):
    lens, H, chunks = LEVELS[name]
    p = U.Paged(lens, 1, 16, dtype, seed=len(name))
    q = rows(1, H)
    got, left = single(p, q)
    assert left == chunks
    U.check(got, *p.answer(q, [1], True, U.DH ** -0.5), name)


@pytest.mark.parametrize("dtype", ["bf16", "e4m3"])
@pytest.mark.parametrize("lens,chunks", [([300000, 280000], 261 + 244), ([600000], 507), ([3 * 8192, 5000, 1, 700], None)])
def test_three_levels(lens, chunks, dtype):
    """261 chunks: 16 groups of 16 and one chunk left over, then 16 groups and that one, then
    two. 507: 32 groups, two, one. Counts: with w half the keys of all sequences and L =
    w / 512 + 1, a sequence of n keys has n / (2 L) chunks, rounded up to whole tiles of 32."""
    p = long_cache(lens, 1, 256, dtype, seed=6)
    q = rows(len(lens), 3, spread=3.0)
    got, left = single(p, q)
    if chunks is not None:
        L = int(sum(lens) / 2 / 512) + 1
        n = [m // (2 * L) for m in lens]
        chunk = [-(-(-(-m // c)) // 32) * 32 for m, c in zip(lens, n)]
        assert left == chunks == sum(-(-m // c) for m, c in zip(lens, chunk))
    # scores up to three times those of TOL's derivation
    want, top = p.answer(q, [1] * len(lens), True, U.DH ** -0.5)
    U.check(got, want, top * (1 + 3 * 2.0 ** -10 / U.TOL))


CASES = {
    "edges": ([1, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 129, 0], 12, 2),
    "cut": ([641, 2050, 777], 28, 4),
    "mha": ([700, 300, 129], 4, 4),
    "mqa": ([900, 257], 8, 1),
    "odd_group": ([333, 6000, 5], 20, 4),
    "one_head": ([1333, 70], 1, 1),
    "many": ([9, 2000, 31] * 40, 10, 2),        # four sequences a lane
}


@pytest.mark.parametrize("page", [16, 32, 128, 256])
@pytest.mark.parametrize("dtype", ["bf16", "e4m3"])
@pytest.mark.parametrize("name", CASES)
def test_against_oracle(name, dtype, page):
    lens, H, Hkv = CASES[name]
    p = U.Paged(lens, Hkv, page, dtype, seed=len(name), extra_cols=512 // page, scales=page != 32)
    for causal in (True, False):
        q = rows(len(lens), H, seed=page)
        got, left = single(p, q, causal=causal)
        assert (left > 0) == (max(lens) >= 640)
        U.check(got, *p.answer(q, [1] * len(lens), causal, U.DH ** -0.5), name)


def test_rows_that_belong_to_no_sequence():
    """q may have a row for every sequence while some have none; what is behind stays."""
    lens, new = [700, 1300, 40, 0, 9], [1, 0, 1, 1, 0]
    p = U.Paged(lens, 2, 16, "bf16", seed=3)
    q = rows(3, 12)
    got, _ = single(p, q, new=new, pad=2)
    U.check(got, *p.answer(q, new, True, U.DH ** -0.5))


@pytest.mark.parametrize("lens", [[20011], [128 * 33 * 3 + 5, 700]])
@pytest.mark.parametrize("dtype", ["bf16", "e4m3"])
def test_windows_of_page_numbers(lens, dtype):
    """Shared by so many sequences that none is cut: a wave's tiles pass 4096 keys, after which
    it loads page numbers again."""
    B = 256
    p = long_cache([lens[b % len(lens)] for b in range(B)], 4, 16, dtype, seed=8)
    q = rows(B, 4)
    got, left = single(p, q)
    assert left == 0
    k, v = p.k_used, p.v_used
    for b in (0, 1, 101, B - 1):
        p.k_used, p.v_used = k[b:b + 1], v[b:b + 1]
        U.check(got[b:b + 1], *p.answer(q[b:b + 1], [1], True, U.DH ** -0.5))


@pytest.mark.parametrize("dtype", ["bf16", "e4m3"])
@pytest.mark.parametrize("lens,new", [([40, 60], [3, 0]), ([2777, 40] + [0] * 40, [30, 1] + [0] * 40)])
def test_unseen_values_have_no_influence(lens, new, dtype):
    """Several rows of one sequence among the single tokens: NaN and infinities behind a row's
    mask; rows that see them get NaN or infinity."""
    lens, new = lens + [0] * sum(new), new + [0] * sum(new)
    p = U.Paged(lens, 2, 16, dtype, seed=9)
    k, v = [x.copy() for x in p.k], [x.copy() for x in p.v]
    m, n = lens[0], new[0]
    for i, bad in ((n - 1, np.nan), (n // 2, np.inf), (n // 3, -np.inf)):
        v[0][m - n + i, :, 7 + i] = bad
    k[0][m - 1, 0, 3] = np.nan
    p = U.Paged(lens, 2, 16, dtype, seed=9, k=k, v=v)
    q = rows(sum(new), 14)
    want, top = p.answer(q, new, True, U.DH ** -0.5)
    got, _ = single(p, q, new=new)
    inf = np.isinf(want)
    assert np.array_equal(np.isposinf(got), np.isposinf(want)) and np.array_equal(np.isneginf(got), np.isneginf(want))
    U.check(np.where(inf, 0.0, got), np.where(inf, 0.0, want), top)
    assert np.isnan(want).any() and not np.isnan(want[0]).any() and not np.isnan(want[n:]).any()


@pytest.mark.parametrize("dtype", ["bf16", "e4m3"])
def test_a_page_that_is_none_reads_as_zeros(dtype):
    p = U.Paged([2000, 90, 20], 2, 16, dtype, seed=11)
    for b, col, bad in ((0, 3, -1), (0, 124, p.n_pages), (0, 125, -7), (1, 0, -(1 << 31)), (2, 1, 1 << 30)):
        p.table[b, col] = bad
        for x in (p.k_used[b], p.v_used[b]):
            x[col * 16:col * 16 + 16] = 0.0
    q = rows(3, 12)
    got, _ = single(p, q)
    U.check(got, *p.answer(q, [1] * 3, True, U.DH ** -0.5))


def test_infinite_scores_touch_their_row_only():
    """Keys whose score is -infinity weigh nothing, whole chunks of them too; a row with one of
    +infinity, or with nothing but -infinity, is NaN; heads and sequences beside it are not."""
    lens = [2050, 2050, 9000, 77, 500]
    p = U.Paged(lens, 2, 16, "bf16", seed=12)
    k = [x.copy() for x in p.k]
    k[0][:1100, 0, 0] = -np.inf  # several whole chunks
    k[1][1234, 0, 0] = np.inf    # one key of a chunk in the middle
    k[2][4000:, 1, 0] = -np.inf
    k[4][:, 0, 0] = -np.inf      # all of it
    p = U.Paged(lens, 2, 16, "bf16", seed=12, k=k)
    q = rows(5, 12)
    q[:, :, 0] = np.abs(q[:, :, 0]) + 0.5
    q[0, 1, 0], q[1, 2, 0] = -1.0, -1.0  # +infinity, and -infinity for one key
    want, top = p.answer(q, [1] * 5, True, U.DH ** -0.5)
    bad = np.isnan(want).all(2)
    assert bad.tolist() == [[h == 1 for h in range(12)], [h < 6 and h != 2 for h in range(12)], [False] * 12, [False] * 12,
                            [h < 6 for h in range(12)]]
    got, _ = single(p, q)
    U.check(got, want, top)


@pytest.mark.parametrize("dtype", ["bf16", "e4m3"])
def test_calls_in_flight_on_two_streams(dtype):
    """No wait between the calls, and no workspace given: each stream's scratch is its own."""
    import torch
    import paper_2608_29291_amd as ce
    work = []
    for i, (lens, new) in enumerate((([9000, 700, 20011], [1, 1, 1]), ([3000, 2000], [150, 1]))):
        p = U.Paged(lens, 2, 16, dtype, seed=20 + i)
        q = rows(sum(new), 12, seed=i)
        c, qd = p.cache(), torch.from_numpy(q).to(torch.bfloat16).cuda()
        off, ln, o = i32([0] + np.cumsum(new).tolist()), i32(lens), [torch.full_like(qd, 77.0) for _ in range(16)]
        work.append((p, q, new, c, qd, off, ln, o, torch.cuda.Stream()))
    torch.cuda.synchronize()
    for r in range(16):
        for p, q, new, c, qd, off, ln, o, st in work:
            ce.ce_paged_attention(c, qd, o[r], off, ln, True, U.DH ** -0.5, stream=st)
    torch.cuda.synchronize()
    for p, q, new, c, qd, off, ln, o, st in work:
        U.check(o[0].float().cpu().numpy(), *p.answer(q, new, True, U.DH ** -0.5))
        for x in o[1:]:
            assert torch.equal(x, o[0])

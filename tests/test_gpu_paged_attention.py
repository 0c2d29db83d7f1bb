"""Attention over the paged cache against the float64 oracle: page sizes, both
page types, head groupings, one token to long caches, chunks and mixed batches,
masks that leave a row empty, and values that must not have any influence."""
import numpy as np
import pytest

import paged_util as U

pytestmark = pytest.mark.gpu


def rows(new, heads, seed=1, spread=1.0):
    rng = np.random.default_rng(seed)
    return U.bf16(rng.standard_normal((sum(new), heads, U.DH)) * spread)


# new rows and cached tokens (the new ones included) of every sequence; query and
# key/value heads
CASES = {
    "one": ([1], [1], 12, 2),
    "edges": ([1] * 12, [1, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 129], 12, 2),
    "decode_cut": ([1] * 3, [513, 2050, 777], 28, 4),
    "decode_mha": ([1, 1, 1], [700, 300, 129], 4, 4),
    "decode_mqa": ([1, 1], [900, 257], 32, 1),
    "drafts": ([4, 1, 5, 2, 0, 1, 3], [900, 1300, 700, 2, 400, 0, 333], 28, 4),
    "row_tiles": ([11, 18, 19, 37], [11, 300, 64, 1100], 28, 4),  # 77, 126, 133 and 259 rows
    "chunk": ([130], [1500], 12, 2),
    "prefill": ([97, 1, 64], [97, 1, 64], 12, 2),
    "mixed": ([150] + [1] * 10 + [0, 33], [700] + [260] * 10 + [50, 33], 28, 4),
    "more_queries": ([5, 40, 3], [2, 7, 0], 12, 2),  # rows that see no key
    "odd_group": ([9, 1], [333, 600], 20, 4),
    "one_head": ([70, 1], [200, 70], 1, 1),
}


@pytest.mark.parametrize("dtype", ["bf16", "e4m3"])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("name", CASES)
def test_against_oracle(name, causal, dtype):
    new, lens, H, Hkv = CASES[name]
    page = [16, 32, 64, 128, 256][sum(map(ord, name)) % 5]
    p = U.Paged(lens, Hkv, page, dtype, seed=len(name))
    q = rows(new, H)
    worst = U.check(U.attend(p, q, new, causal), *p.answer(q, new, causal, U.DH ** -0.5), name)
    print(f"[paged] {name} page {page} {dtype} causal {causal}: {worst:.2f} of the tolerance", flush=True)


@pytest.mark.parametrize("page", [16, 32, 64, 128, 256])
@pytest.mark.parametrize("dtype", ["bf16", "e4m3"])
def test_page_sizes(page, dtype):
    new, lens = [1, 90, 1, 6], [page, 3 * page + 5, 2 * page - 1, 1030]
    p = U.Paged(lens, 2, page, dtype, seed=page)
    q = rows(new, 12)
    U.check(U.attend(p, q, new, True), *p.answer(q, new, True, U.DH ** -0.5))


@pytest.mark.parametrize("B", [64, 65, 255, 256, 257, 700])
def test_many_sequences(B):
    """One wave plans up to 64 and up to 256 sequences, a launch of its own more."""
    rng = np.random.default_rng(B)
    new = [int(x) for x in rng.choice([0, 1, 1, 1, 2, 7], B)]
    new[B // 2] = 40
    lens = [int(n + rng.integers(0, 30)) for n in new]
    lens[B - 1], lens[B // 3] = 1300, 900
    p = U.Paged(lens, 2, 16, "bf16", seed=B)
    q = rows(new, 4)
    U.check(U.attend(p, q, new, True), *p.answer(q, new, True, U.DH ** -0.5))


@pytest.mark.parametrize("dtype", ["bf16", "e4m3"])
def test_long_cache(dtype):
    """Many chunks, combined in eight parts; page numbers reloaded on the way."""
    new, lens = [1, 20], [20011, 9000]
    p = U.Paged(lens, 1, 16, dtype, seed=3)
    q = rows(new, 7)
    U.check(U.attend(p, q, new, True), *p.answer(q, new, True, U.DH ** -0.5))


@pytest.mark.parametrize("dtype", ["bf16", "e4m3"])
def test_long_caches_of_single_tokens(dtype):
    """More than 16 chunks: they meet in two levels, in groups of 16 and a rest."""
    lens = [20011, 9000, 8193, 1]
    p = U.Paged(lens, 1, 16, dtype, seed=5)
    q = rows([1] * 4, 7)
    U.check(U.attend(p, q, [1] * 4, True), *p.answer(q, [1] * 4, True, U.DH ** -0.5))


def test_more_than_256_chunks_of_one_token():
    """Three levels: one head over 600000 keys, the same 32 pages over and over."""
    p = U.Paged([32 * 256], 1, 256, "bf16", seed=6)
    times = 600000 // (32 * 256) + 1
    p.table = np.concatenate([np.tile(p.table[:, :32], (1, times)), p.table[:, 32:]], 1)
    p.lens = [600000]
    p.k_used, p.v_used = ([np.tile(x[0], (times, 1, 1))[:600000]] for x in (p.k, p.v))
    q = rows([1], 3, spread=3.0)
    got, (want, top) = U.attend(p, q, [1], True), p.answer(q, [1], True, U.DH ** -0.5)
    U.check(got, want, top)


@pytest.mark.parametrize("dtype", ["bf16", "e4m3"])
@pytest.mark.parametrize("n", [1, 40])
def test_shared_pages_and_long_chunks(n, dtype):
    """So many sequences over one long prefix that none is cut: a workgroup's keys run
    over several windows of page numbers."""
    B, Hkv, H = 140, 4, 16
    p = U.Paged([8500], Hkv, 16, dtype, seed=4)
    p.table, p.lens = np.repeat(p.table, B, 0), [8500 - 8 * (b % 3) for b in range(B)]
    q = rows([n] * B, H)
    got = U.attend(p, q, [n] * B, True)
    k, v = p.k_used[0], p.v_used[0]
    for b in (0, 1, 77, B - 1):
        p.k_used, p.v_used = [k[:p.lens[b]]], [v[:p.lens[b]]]
        sel = slice(b * n, b * n + n)
        U.check(got[sel], *p.answer(q[sel], [n], True, U.DH ** -0.5))


@pytest.mark.parametrize("new,lens,H,Hkv", [([3, 2], [40, 700], 7, 1), ([60, 130], [200, 1400], 7, 1)])
@pytest.mark.parametrize("dtype", ["bf16", "e4m3"])
def test_unseen_values_have_no_influence(new, lens, H, Hkv, dtype):
    """NaN and infinities in keys and values behind a query's mask; rows that see them get NaN."""
    p = U.Paged(lens, Hkv, 16, dtype, seed=8)
    k = [x.copy() for x in p.k]
    v = [x.copy() for x in p.v]
    for b, (n, m) in enumerate(zip(new, lens)):
        for i, bad in ((n - 1, np.nan), (n // 2, np.inf), (n // 3, -np.inf)):
            v[b][m - n + i, :, 5 + i % 50] = bad
        k[b][m - 1, 0, 3] = np.nan
    p = U.Paged(lens, Hkv, 16, dtype, seed=8, k=k, v=v)
    q = rows(new, H)
    with np.errstate(invalid="ignore"):
        want, top = p.answer(q, new, True, U.DH ** -0.5)
    got = U.attend(p, q, new, True)
    inf = np.isinf(want)
    assert np.array_equal(np.isposinf(got), np.isposinf(want)) and np.array_equal(np.isneginf(got), np.isneginf(want))
    U.check(np.where(inf, 0.0, got), np.where(inf, 0.0, want), top)
    assert np.isnan(want).any() and not np.isnan(want[0]).any()


@pytest.mark.parametrize("new,lens", [([1], [600]), ([80], [90])])
def test_scores_without_a_finite_maximum(new, lens):
    """All scores -infinity are 0 / 0; one +infinity is NaN; neither touches other rows."""
    p = U.Paged(lens, 1, 32, "bf16", seed=9)
    k = [x.copy() for x in p.k]
    k[0][:, 0, 0] = -np.inf
    p = U.Paged(lens, 1, 32, "bf16", seed=9, k=k)
    q = np.abs(rows(new, 2)) + 0.5
    q[:, 1, 0] = -q[:, 1, 0]
    got = U.attend(p, q, new, True)
    assert np.isnan(got).all()


def test_sharp_scores():
    """One key far above the rest: the maximum moves by hundreds along the cache."""
    new, lens = [2, 50], [1500, 400]
    p = U.Paged(lens, 2, 16, "bf16", seed=10)
    q = rows(new, 12, spread=12.0)
    # scores up to 500: their fp32 error is twelve times that of TOL's derivation
    got, (want, top) = U.attend(p, q, new, True), p.answer(q, new, True, U.DH ** -0.5)
    U.check(got, want, top * (1 + 12 * 2.0 ** -10 / U.TOL))


def test_a_page_that_is_none_reads_as_zeros():
    for new, lens in (([1, 2], [200, 90]), ([60, 30], [200, 90])):
        for dtype in ("bf16", "e4m3"):
            p = U.Paged(lens, 2, 16, dtype, seed=11)
            for b, col, bad in ((0, 3, -1), (0, 12, p.n_pages), (1, 0, -(1 << 31))):
                p.table[b, col] = bad
                lo, hi = col * 16, min(col * 16 + 16, lens[b])
                for x in (p.k_used[b], p.v_used[b]):
                    x[lo:hi] = 0.0
            q = rows(new, 12)
            U.check(U.attend(p, q, new, True), *p.answer(q, new, True, U.DH ** -0.5))


def test_strides_and_interleaved_layers():
    """q as a part of a fused projection's rows, pages of two layers in one allocation."""
    import torch
    import paper_2608_29291_amd as ce
    new, lens, H, Hkv = [1, 40], [300, 500], 12, 2
    p = U.Paged(lens, Hkv, 32, "bf16", seed=12)
    q = rows(new, H)
    c = p.cache()
    pool = torch.full((p.n_pages, 2, 2, Hkv, 32, U.DH), float("nan"), dtype=torch.bfloat16, device="cuda")
    pool[:, 1, 0], pool[:, 1, 1] = c.k, c.v
    c = ce.KVCache(pool[:, 1, 0], pool[:, 1, 1], c.page_table)
    qkv = torch.full((sum(new), H + 2 * Hkv, U.DH), float("nan"), dtype=torch.bfloat16, device="cuda")
    qkv[:, :H] = torch.from_numpy(q).to(torch.bfloat16).cuda()
    o = torch.empty(sum(new), H, U.DH, dtype=torch.bfloat16, device="cuda")
    off = torch.tensor([0, 1, 41], dtype=torch.int32).cuda()
    ce.ce_paged_attention(c, qkv[:, :H], o, off, torch.tensor(lens, dtype=torch.int32).cuda(), True, U.DH ** -0.5)
    torch.cuda.synchronize()
    U.check(o.float().cpu().numpy(), *p.answer(q, new, True, U.DH ** -0.5))


def test_runs_repeat_bit_for_bit():
    new, lens = [1, 200, 3], [5000, 1300, 900]
    p = U.Paged(lens, 2, 16, "bf16", seed=13)
    q = rows(new, 12)
    first = U.attend(p, q, new, True)
    for ws in (True, False):
        assert np.array_equal(U.attend(p, q, new, True, ws=ws), first)


def test_bad_lengths_and_offsets_stay_in_bounds():
    """Lengths past the table are clamped; offsets out of order give some answer."""
    import torch
    import paper_2608_29291_amd as ce
    p = U.Paged([100, 200, 50], 2, 16, "bf16", seed=14)
    c = p.cache()
    q = torch.randn(300, 4, U.DH, dtype=torch.bfloat16, device="cuda")
    o = torch.empty_like(q)
    for off in ([0, 300, 100, 300], [-5, 1 << 30, 3, 2], [300, 0, 300, 0]):
        for lens in ([1 << 30, -3, 7], [100, 200, 50]):
            ce.ce_paged_attention(c, q, o, torch.tensor(off, dtype=torch.int32).cuda(),
                                  torch.tensor(lens, dtype=torch.int32).cuda(), True, U.DH ** -0.5)
    torch.cuda.synchronize()

"""Verification of drafted tokens against the float64 oracle: all outputs are whole numbers and equal."""
import numpy as np
import pytest
import torch

import draft_util as du
from oracle import draft as od

pytestmark = pytest.mark.gpu
ce = pytest.importorskip("paper_2608_29291_amd")


class Case:
    """Trees whose drafted tokens are likely ones (or drawn from `probs`)."""

    def __init__(self, new, vocab, dtype, drawn=False, chains=False, temps=None, seed=0, spread=2.0):
        rng = np.random.default_rng(seed)
        self.rng, self.new, self.vocab, self.dtype = rng, new, vocab, dtype
        n = sum(new)
        self.off = du.offsets(new)
        self.parents = [list(range(-1, k - 1)) if chains else du.tree(rng, k, 0.5) if k else [] for k in new]
        x = rng.standard_normal((n, vocab)) * spread
        self.tokens = rng.integers(0, vocab, n)
        self.probs = None
        if drawn:
            y = x + rng.standard_normal((n, vocab))
            q = np.exp(y - y.max(-1, keepdims=True))
            self.probs = (q / q.sum(-1, keepdims=True)).astype(np.float32)
        for b, t in enumerate(self.parents):
            for i, p in enumerate(t):
                if p >= 0:
                    r = self.off[b] + p
                    if drawn:
                        self.tokens[self.off[b] + i] = rng.choice(vocab, p=self.probs[r] / self.probs[r].sum(dtype=np.float64))
                    else:
                        x[r, self.tokens[self.off[b] + i]] = np.log(vocab) + spread + rng.standard_normal()
        self.logits = torch.from_numpy(x.astype(np.float32)).to(dtype)
        self.temps = np.ones(len(new), np.float32) if temps is None else np.array(temps, np.float32)
        self.us, self.ua = rng.random(n).astype(np.float32), rng.random(n).astype(np.float32)

    def answer(self):
        x = self.logits.double().numpy()
        kept = np.full(len(x), -1, np.int32)
        n_kept, nxt = [], []
        for b, n in enumerate(self.new):
            s = slice(self.off[b], self.off[b] + n)
            walk, t = od.verify(self.parents[b], self.tokens[s], x[s], float(self.temps[b]), self.us[s],
                                None if self.probs is None else self.probs[s], self.ua[s])
            kept[self.off[b]:self.off[b] + len(walk)] = walk
            n_kept.append(len(walk))
            nxt.append(t)
        return kept, n_kept, nxt

    def run(self, parents=True, temps=True, ws=True, stream=None, logits=None, probs=None, pad=3, rest=True, fill=0xff):
        n = len(self.tokens)
        flat = [p for t in self.parents for p in t]
        i32 = lambda x: du.up(np.concatenate([np.array(x, np.int32), np.zeros(pad, np.int32)]))
        f32 = lambda x: du.up(np.concatenate([x, np.full(pad, 0.5, np.float32)]))
        d = ce.Drafts(du.up(self.off), i32(flat) if parents else None, i32(self.tokens))
        grown = lambda x: torch.cat([x, torch.zeros((pad, x.shape[1]), dtype=x.dtype)]).cuda()
        logits = grown(self.logits) if logits is None else logits
        if self.probs is not None and probs is None:
            probs = grown(torch.from_numpy(self.probs))
        B = len(self.new)
        kept = torch.full((n + pad,), 55, dtype=torch.int32, device="cuda")
        nk, nxt = (torch.full((B,), -9, dtype=torch.int32, device="cuda") for _ in range(2))
        w = None
        if ws:
            w = ce.alloc_verify_workspace(d, logits.shape[1], probs is not None)
            w.fill_(fill)  # what is on entry must not matter
        torch.cuda.synchronize()
        ce.ce_verify_drafts(d, logits, f32(self.us), kept, nk, nxt, temperature=du.up(self.temps) if temps else None,
                            draft_probs=probs, u_accept=f32(self.ua) if probs is not None else None, ws=w, stream=stream)
        torch.cuda.synchronize()
        kept = kept.cpu().numpy()
        assert not rest or (kept[n:] == 55).all(), "rows behind the last were written"
        return kept[:n], nk.tolist(), nxt.tolist()

    def check(self, **kw):
        got, want = self.run(**kw), self.answer()
        np.testing.assert_array_equal(got[0], want[0])
        assert got[1] == want[1] and got[2] == want[2]
        return want


DTYPES = [torch.bfloat16, torch.float32]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("vocab", [1, 2, 5, 255, 1000, 4095, 4096, 4097, 8200, 50001])
def test_chosen_drafts(dtype, vocab):
    temps = [1.0, 0.0, 0.7, 1.3, -1.0, np.nan, 0.05]
    c = Case([9, 26, 1, 70, 12, 5, 130 if vocab < 5000 else 8], vocab, dtype, temps=temps, seed=vocab)
    _, n_kept, _ = c.check()
    assert vocab < 5 or max(n_kept) > 1


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("chains", [True, False])
@pytest.mark.parametrize("vocab", [1, 3, 40, 4096, 4099, 20001])
def test_drawn_drafts(dtype, chains, vocab):
    temps = [1.0, 0.0, 0.9, 1.1, 1.0, 0.8]
    total = 0
    for seed in range(4):
        c = Case([9, 6, 30, 1, 40, 0], vocab, dtype, drawn=True, chains=chains, temps=temps, seed=seed)
        total += sum(c.check()[1])
    assert vocab == 1 or total > 24  # some are accepted


def test_many_siblings_are_rejected_one_after_another():
    # one row with 60 children whose tokens the target hardly has: a pass over the row for each
    c = Case([61, 20, 61], 9000, torch.float32, drawn=True, seed=3)
    for b in (0, 2):
        c.parents[b] = [-1] + [0] * 60
        r = c.off[b]
        for i in range(1, 61):
            c.tokens[r + i] = c.rng.choice(9000, p=c.probs[r] / c.probs[r].sum(dtype=np.float64))
        c.logits[r, torch.from_numpy(c.tokens[r + 1:r + 40])] = -8.0
    c.check()


def test_a_later_sibling_is_accepted_and_the_walk_goes_on():
    hit = 0
    for seed in range(12):
        c = Case([30] * 4, 50, torch.float32, drawn=True, seed=seed, spread=0.5)
        c.ua[:] = np.where(c.rng.random(len(c.ua)) < 0.5, 0.999, c.ua)
        kept, n_kept, _ = c.check()
        for b in range(4):
            for j in range(1, n_kept[b]):
                i, p = kept[c.off[b] + j], kept[c.off[b] + j - 1]
                hit += c.parents[b].index(p) != i
    assert hit > 3


@pytest.mark.parametrize("drawn", [False, True])
@pytest.mark.parametrize("vocab", [262145, 1300001])
def test_more_tokens_than_a_wave_holds_chunks_of(vocab, drawn):
    # the row's whole is spread evenly, so its token lies in any chunk
    c = Case([5, 4], vocab, torch.float32, drawn=drawn, seed=vocab, spread=0.5)
    c.us[:] = np.linspace(0.05, 0.95, len(c.us))
    c.check()


@pytest.mark.parametrize("B,n", [(1, 1), (65, 2), (300, 3), (5000, 1)])
def test_batches(B, n):
    new = [n if b % 7 else 0 for b in range(B)]
    new[-1] = n
    Case(new, 300, torch.bfloat16, seed=B).check()


@pytest.mark.parametrize("drawn", [False, True])
@pytest.mark.parametrize("B", [1, 3, 64, 100])
def test_batches_that_are_mostly_padding(B, drawn):
    # (more rows behind the last sequence than all of the chip's waves take at once)
    c = Case([3, 0, 5, 1][:B] * (B // 4 + 1), 2100, torch.bfloat16, drawn=drawn, seed=B)
    c.check(pad=7000)


def test_chains_without_parents_and_no_temperature():
    c = Case([7, 1, 0, 20], 700, torch.bfloat16, chains=True)
    c.check(parents=False, temps=False)
    Case([7, 1, 0, 20], 700, torch.float32, drawn=True, chains=True, seed=2).check(parents=False, temps=False)


@pytest.mark.parametrize("dtype", DTYPES)
def test_spaced_and_unaligned_rows(dtype):
    c = Case([9, 30], 1003, dtype, drawn=True)
    n = len(c.tokens) + 3
    big = torch.full((n, 1050), 30.0, dtype=dtype, device="cuda")
    view = big[:, 7:1010]
    view[:n - 3] = c.logits.cuda()
    probs = torch.full((n, 1021), 0.9, device="cuda")
    pv = probs[:, 5:1008]
    pv[:n - 3] = torch.from_numpy(c.probs).cuda()
    c.check(logits=view, probs=pv)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("drawn", [False, True])
def test_special_logits(dtype, drawn):
    inf, nan = float("inf"), float("nan")
    c = Case([4] * 7, 5000, dtype, drawn=drawn, temps=[1, 1, 0, 1, 1, 0.5, 0], chains=True)
    x = c.logits
    x[0] = nan
    x[4, ::2] = -inf
    x[4, 3000:] = nan
    x[8, 100] = x[8, 4500] = 1e30  # ties of the largest: the lowest
    x[12:16] = -inf
    x[13, 17] = -3.0  # one token only
    x[12, [7, 4097, 4999]] = inf  # these three share it
    x[16] = 3e38
    x[20, 11] = 3e38
    x[24] = -inf
    if drawn:
        c.probs[0, :] = nan
        c.probs[4, ::3] = nan
        c.probs[12] = 0.0
        c.probs[20, :2500] = -1.0
    c.check()


def test_numbers_at_their_ends():
    c = Case([5, 5, 5], 4100, torch.float32, chains=True)
    c.us[:] = [0.0] * 5 + [1.0 - 2.0 ** -24] * 5 + [1.0] * 5
    c.logits[:, :10] = -float("inf")
    c.logits[:, -10:] = -float("inf")
    c.check()
    c = Case([5, 5, 5], 4100, torch.float32, chains=True, drawn=True)
    c.ua[:] = [0.0] * 5 + [1.0 - 2.0 ** -24] * 5 + [1.0] * 5
    c.check()


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("offset,temp", [(0.0, 1.0), (3e4, 0.01), (-3e5, 0.05), (2e6, 0.3), (2e7, 1.0), (-1e12, 1.0), (1e30, 2.0),
                                         (5.0, 1e-38), (5.0, 3e38), (5.0, float("inf")), (0.0, 1e-45)])
def test_hidden_chunks_and_far_logits(dtype, offset, temp):
    # whole chunks of hidden tokens at both ends, numbers at theirs, and logits and temperatures of any size
    c = Case([4, 4, 4, 4], 9000, dtype, chains=True, temps=[temp] * 4)
    c.us[:] = [0.0] * 4 + [1.0 - 2.0 ** -24] * 4 + [0.3] * 8
    x = c.logits.float() * (1.0 if abs(offset) < 1e5 else abs(offset) * 2.0 ** -9) + offset
    x[:, :5000] = -float("inf")
    x[:, 8000:] = -float("inf")
    x[2, 8500] = float("nan")
    x[3, 5100:7900] = offset - abs(offset) - 2e4  # far below the others
    c.logits = x.to(dtype)
    c.check()


def test_equal_distributions_and_tokens_of_no_vocabulary():
    c = Case([6, 6, 6], 600, torch.float32, drawn=True, chains=False, seed=5)
    c.parents = [[-1, 0, 0, 0, 1, 1]] * 3
    x = c.logits.double().numpy()
    p = np.exp(x - x.max(-1, keepdims=True))
    c.probs = (p / p.sum(-1, keepdims=True)).astype(np.float32)
    c.ua[:] = 0.999
    c.tokens[[1, 8]] = [-1, 600]  # not asked
    c.tokens[13] = 2 ** 30
    c.check()
    c.probs = None
    c.check()
    # all weight of the draft on one token that the target does not have
    c = Case([3], 64, torch.float32, drawn=True, chains=True)
    c.logits[0, 5] = -float("inf")
    c.probs[0] = 0.0
    c.probs[0, 5] = 1.0
    c.tokens[1] = 5
    c.check()


def test_flat_rows_of_many_tokens_have_borders_close_together():
    # 1e5 equal weights and one that is as large as all others: 32-bit sums would be off by many tokens
    c = Case([3] * 8, 100003, torch.float32, chains=True, spread=0.0)
    c.logits[:] = 0.25
    c.logits[:, 7] = 0.25 + float(np.log(1e5))
    c.check()


def test_repeats_streams_and_scratch():
    for drawn in (False, True):
        c = Case([20, 33, 5], 9001, torch.bfloat16, drawn=drawn, seed=8)
        c.check()
        c.check(ws=False)
        c.check(stream=torch.cuda.Stream())
        c.check(ws=False, stream=torch.cuda.Stream())


@pytest.mark.parametrize("drawn", [False, True])
def test_one_workspace_for_calls_of_many_kinds(drawn):
    # what a call leaves in its workspace is any content to the next
    cases = [Case(new, vocab, torch.bfloat16, drawn=drawn, seed=i)
             for i, (new, vocab) in enumerate([([9, 3], 7000), ([5] * 70, 500), ([1], 30000), ([9, 0, 3], 7000)])]
    ws = torch.full((1 << 22,), 0x5a, dtype=torch.uint8, device="cuda")
    for _ in range(3):
        for c in cases:
            want, n = c.answer(), len(c.tokens)
            i32 = lambda x: du.up(np.array(x, np.int32))
            kept, nk, nxt = i32([55] * n), i32([-9] * len(c.new)), i32([-9] * len(c.new))
            ce.ce_verify_drafts(ce.Drafts(du.up(c.off), i32([p for t in c.parents for p in t]), i32(c.tokens)), c.logits.cuda(),
                                du.up(c.us), kept, nk, nxt, draft_probs=du.up(c.probs) if drawn else None,
                                u_accept=du.up(c.ua) if drawn else None, ws=ws)
            np.testing.assert_array_equal(kept.cpu().numpy(), want[0])
            assert nk.tolist() == want[1] and nxt.tolist() == want[2]


def test_offsets_out_of_order_stay_in_bounds():
    c = Case([10, 10, 10], 500, torch.float32, drawn=True)
    want = c.answer()
    for off in ([0, 25, 5, 30], [-3, 10, 20, 1 << 30], [7, 7, 7, 7], [30, 20, 10, 0]):
        c.off = np.array(off, np.int32)
        for pad in (3, 5000):
            for fill in (0xff, 0):
                kept, n_kept, _ = c.run(rest=False, pad=pad, fill=fill)
                # (a sequence whose rows are not its own has no walk: its outputs stay as they were)
                assert all(k == -9 or 0 <= k <= len(c.tokens) + pad for k in n_kept), n_kept
                assert ((kept == 55) | (kept == -1) | ((kept >= 0) & (kept < len(c.tokens) + pad))).all()
    c.off = du.offsets(c.new)
    got = c.run()
    np.testing.assert_array_equal(got[0], want[0])


def test_refusals_of_the_binding():
    c = Case([3], 50, torch.float32)
    i = torch.zeros(3, dtype=torch.int32, device="cuda")
    u, x = torch.zeros(3, device="cuda"), torch.zeros((3, 50), device="cuda")
    d = ce.Drafts(du.up(du.offsets([3])), i, i)
    args = (u, i, i[:1], i[:1])
    for d2, y, kw in ((ce.Drafts(d.offsets, i), x, {}), (d, x[:2], {}), (d, x.t(), {}), (d, x.half(), {}), (d, x.cpu(), {}),
                      (d, x, {"draft_probs": x[:, :49], "u_accept": u}), (d, x, {"temperature": u.double()})):
        with pytest.raises(ValueError):
            ce.ce_verify_drafts(d2, y, *args, **kw)
    for kw in ({"draft_probs": x}, {"u_accept": u}, {"ws": torch.zeros(256, dtype=torch.uint8, device="cuda")}):
        with pytest.raises(ce.CERouterError):
            ce.ce_verify_drafts(d, x, *args, **kw)

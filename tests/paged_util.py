"""Helpers of the paged cache's tests: caches built from dense keys and values,
and the float64 answer. Test infrastructure only."""
import numpy as np
import torch

from oracle import paged as op

DH = 128


def quantize(x, scale):
    """Codes of x [..., H_kv, dh] / scale [H_kv] in the 8-bit format (one float32 division)."""
    y = np.asarray(x, np.float32) / np.asarray(scale, np.float32)[:, None]
    return op.e4m3(y)


def bf16(x):
    """x rounded to bf16, as float32."""
    return torch.from_numpy(np.asarray(x, np.float32)).to(torch.bfloat16).float().numpy()


class Paged:
    """Sequences of given lengths in shuffled pages. What no call may use is filled
    with `poison` (rows behind a sequence's end, free pages) or nonsense (table
    entries behind its last page)."""

    def __init__(self, lens, heads_kv, page, dtype, seed=0, k=None, v=None, poison=float("nan"), spread=1.0, spare=2,
                 extra_cols=2, scales=True):
        rng = np.random.default_rng(seed)
        self.lens, self.page, self.dtype, self.hkv = list(lens), page, dtype, heads_kv
        held = [-(-n // page) for n in self.lens]
        self.n_pages = sum(held) + spare
        self.width = max(held + [0]) + extra_cols
        order = rng.permutation(self.n_pages)
        self.table = np.full((len(self.lens), self.width), 1 << 30, np.int32)
        self.k = [bf16(rng.standard_normal((n, heads_kv, DH)) * spread) for n in self.lens] if k is None else k
        self.v = [bf16(rng.standard_normal((n, heads_kv, DH))) for n in self.lens] if v is None else v
        shape = (self.n_pages, heads_kv, page, DH)
        self.ks = self.vs = None
        if dtype == "e4m3":
            if scales:
                self.ks = rng.uniform(0.01, 0.03, heads_kv).astype(np.float32)
                self.vs = rng.uniform(0.01, 0.03, heads_kv).astype(np.float32)
            one = np.ones(heads_kv, np.float32)
            fill = np.uint8(0x7f) if np.isnan(poison) else op.e4m3(poison)
            pools, used = [], []
            for x, s in ((self.k, self.ks), (self.v, self.vs)):
                s = one if s is None else s
                codes = [quantize(y, s) for y in x]
                pools.append(self._fill(np.full(shape, fill, np.uint8), codes, held, order))
                used.append([op.e4m3_value(c) * s.astype(np.float64)[:, None] for c in codes])
            self.pk, self.pv = (torch.from_numpy(p).view(torch.float8_e4m3fn) for p in pools)
            self.k_used, self.v_used = used
        else:
            self.pk, self.pv = (torch.from_numpy(self._fill(np.full(shape, poison, np.float32), x, held, order)).to(
                torch.bfloat16) for x in (self.k, self.v))
            self.k_used, self.v_used = self.k, self.v

    def _fill(self, pool, seqs, held, order):
        at = 0
        for b, x in enumerate(seqs):
            ids = order[at:at + held[b]]
            self.table[b, :held[b]] = ids
            at += held[b]
            for j in range(len(x)):
                pool[ids[j // self.page], :, j % self.page] = x[j]
        self.free = order[at:]
        return pool

    def cache(self):
        import paper_2608_29291_amd as ce
        up = lambda x: None if x is None else torch.from_numpy(x).cuda()
        return ce.KVCache(self.pk.cuda(), self.pv.cuda(), up(self.table), up(self.ks), up(self.vs))

    def answer(self, q, new, causal, scale):
        """float64 outputs of packed rows q and, per row and head, the largest value among the keys seen."""
        out, top, at = np.zeros(q.shape), np.zeros(q.shape[:2]), 0
        g = q.shape[1] // self.hkv
        for b, n in enumerate(new):
            out[at:at + n] = op.attend(q[at:at + n], self.k_used[b], self.v_used[b], causal, scale)
            v = np.abs(np.where(np.isfinite(self.v_used[b]), self.v_used[b], 0.0))
            if len(v):
                top[at:at + n] = np.repeat(v.max((0, 2)), g)[None]
            at += n
        return out, top


def attend(p, q, new, causal, scale=DH ** -0.5, cache=None, ws=True, stream=None):
    """ce_paged_attention on bf16 rows q; rows behind the last one are checked to stay as they were."""
    import paper_2608_29291_amd as ce
    c = cache or p.cache()
    qd = torch.from_numpy(q).to(torch.bfloat16).cuda()
    pad = torch.zeros((3,) + qd.shape[1:], dtype=torch.bfloat16, device="cuda")
    qd = torch.cat([qd, pad])  # a capacity above the packed count
    o = torch.full(qd.shape, 77.0, dtype=torch.bfloat16, device="cuda")
    off = torch.from_numpy(np.concatenate([[0], np.cumsum(new)]).astype(np.int32)).cuda()
    lens = torch.tensor(p.lens, dtype=torch.int32).cuda()
    w = ce.alloc_paged_workspace(c, qd.shape[0], qd.shape[1]) if ws else None
    if w is not None:
        w.fill_(0xff)  # NaN: what is on entry must not matter
    torch.cuda.synchronize()  # (the call may be made on another stream)
    ce.ce_paged_attention(c, qd, o, off, lens, causal, scale, ws=w, stream=stream)
    torch.cuda.synchronize()
    o = o.float().cpu().numpy()
    assert (o[len(q):] == 77.0).all(), "rows behind the last were written"
    return o[:len(q)]


# The probabilities are rounded to bf16 for the product with V (half a step: 2^-8
# of each weight, so of the largest value at most) and the output once more (2^-8 of
# itself). Scores are fp32 sums of 128 products: their error, 128 2^-24 times the
# sum of the products' magnitudes (below 40 for the inputs here), moves a weight by
# 2^-11 at most, a second time through the maximum's fp32 exponent.
TOL = 2 * 2.0 ** -8 + 2.0 ** -10


def check(got, want, top, what=""):
    bad = np.isnan(want)
    assert np.array_equal(np.isnan(got), bad), f"{what}: NaN elsewhere ({np.isnan(got).sum()} and {bad.sum()})"
    err = np.where(bad, 0.0, np.abs(got - np.where(bad, 0.0, want)))
    lim = TOL * top[:, :, None] + 1e-6
    worst = (err / lim).max() if err.size else 0.0
    assert worst <= 1.0, f"{what}: {worst} times the tolerance at {np.unravel_index((err / lim).argmax(), err.shape)}"
    return worst

"""The paged key/value cache of a routed layer -- TEST INFRASTRUCTURE ONLY.

Paper section 3.4, task-adaptive token compaction: the packed keys / values of a
routed layer form the compressed cache that decoding attends to. Here the cache
is kept in pages: token j of sequence b is row j % P of page table[b, j // P].

  reserve -- pages and slots for new rows, one page at a time from a Python list
  e4m3    -- nearest value of the 8-bit format (448 the largest), ties to even
  attend  -- attention over one sequence's keys and values, row by row

Readings taken here: as in the attention oracle a query that sees no key
outputs zeros; every other query follows the formula, so visible NaN come through
and scores that are all -infinity give 0 / 0.
"""
import numpy as np


def reserve(lens, new, page, table, free, reset=None):
    """lens, new: lists of ints; table: int array [B, width]; free: list, its end
    the top of the stack. Returns (lens, start, slots, table, free, refused) with
    refused[b] in {"", "pages", "long"}; the arguments are left as they were."""
    lens, table, free = [int(x) for x in lens], np.array(table), [int(x) for x in free]
    width = table.shape[1]
    for b in range(len(lens)):
        if reset is not None and reset[b]:
            for j in range(-(-lens[b] // page)):
                free.append(int(table[b, j]))
            lens[b] = 0
    start, slots, refused, short = [], [], [], False
    for b, n in enumerate(new):
        n = int(n)
        want = -(-(lens[b] + n) // page) - -(-lens[b] // page)
        why = ""
        if -(-(lens[b] + n) // page) > width:
            why = "long"
        elif want and (short or want > len(free)):
            why, short = "pages", True  # and nobody behind it gets pages
        refused.append(why)
        start.append(-1 if why else lens[b])
        for i in range(n):
            if why:
                slots.append(-1)
                continue
            t = lens[b] + i
            if t % page == 0:
                table[b, t // page] = free.pop()
            slots.append(int(table[b, t // page]) * page + t % page)
        if not why:
            lens[b] += n
    return lens, start, slots, table, free, refused


def _e4m3_values():
    """The 127 values of the format that are not negative, in the order of their codes."""
    out = []
    for code in range(127):
        e, m = code >> 3, code & 7
        out.append(m * 2.0 ** -9 if e == 0 else (8 + m) * 2.0 ** (e - 10))
    return np.array(out)


def e4m3(x):
    """Codes (uint8) of the nearest values to x, limited to +-448; ties to the even code; NaN is 0x7f."""
    x = np.asarray(x, np.float64)
    vals = _e4m3_values()
    a = np.minimum(np.abs(np.nan_to_num(x, nan=0.0, posinf=448.0, neginf=-448.0)), 448.0)
    hi = np.clip(np.searchsorted(vals, a), 0, 126)
    lo = np.maximum(hi - 1, 0)
    d_lo, d_hi = a - vals[lo], vals[hi] - a
    pick = np.where((d_lo < d_hi) | ((d_lo == d_hi) & (lo % 2 == 0)), lo, hi).astype(np.uint8)
    pick = pick | np.where(np.signbit(x), 0x80, 0).astype(np.uint8)
    return np.where(np.isnan(x), np.uint8(0x7f), pick)


def e4m3_value(code):
    code = np.asarray(code, np.uint8)
    vals = np.append(_e4m3_values(), np.nan)
    return np.where(code & 0x80, -1.0, 1.0) * vals[code & 0x7f]


def attend(q, k, v, causal, scale):
    """q [n_q, H, dh], k / v [n_k, H_kv, dh], float64; returns O [n_q, H, dh]. Every
    row uses the keys that it sees and no others."""
    q, k, v = (np.asarray(x, np.float64) for x in (q, k, v))
    n_q, H, _ = q.shape
    n_k, g = k.shape[0], H // k.shape[1]
    out = np.zeros(q.shape)
    with np.errstate(invalid="ignore", over="ignore"):  # NaN and infinities are inputs here
        for i in range(n_q):
            sees = min(max(n_k - n_q + i + 1, 0), n_k) if causal else n_k
            if sees == 0:
                continue
            for h in range(H):
                s = scale * (k[:sees, h // g] @ q[i, h])
                m = np.nan if np.isnan(s).any() else s.max()
                p = np.exp(s - m)
                out[i, h] = (p @ v[:sees, h // g]) / p.sum()
    return out

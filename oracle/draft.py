"""Drafted decoding over the paged cache, and rotary positions -- TEST INFRASTRUCTURE ONLY.

  masks   -- who sees whom in a tree given by parents, and depths
  attend  -- attention over one sequence's keys and values under truth values
  verify  -- the rows of one tree that the target's probabilities accept, row by row
  keep    -- accepted rows moved up in a sequence given as a list
  rotary  -- pairs turned by position times frequency, as complex numbers

Written from the definitions in float64 and with Python's lists; nothing is shared with
the library.
"""
import math

import numpy as np


def masks(parents):
    """([n, n] truth values, depths) of a tree; a parent that is not before its row is none."""
    n = len(parents)
    seen, depth = np.zeros((n, n), bool), np.zeros(n, int)
    for i, p in enumerate(parents):
        if 0 <= p < i:
            seen[i] = seen[p]
            depth[i] = depth[p] + 1
        seen[i, i] = True
    return seen, depth


def words(seen, n_words):
    """Truth values [n, m] as uint32 words [n, n_words], bit j % 32 of word j // 32."""
    n, m = seen.shape
    bits = np.zeros((n, 32 * n_words), np.uint64)
    bits[:, :min(m, 32 * n_words)] = seen[:, :32 * n_words]
    return (bits.reshape(n, n_words, 32) << np.arange(32, dtype=np.uint64)).sum(-1).astype(np.uint32)


def attend(q, k, v, seen, scale):
    """q [n_q, H, dh], k / v [n_k, H_kv, dh], seen [n_q, n_k]. Every row uses the keys that it
    sees and no others; a row that sees none is zeros."""
    q, k, v = (np.asarray(x, np.float64) for x in (q, k, v))
    n_q, H, _ = q.shape
    g = H // k.shape[1]
    out = np.zeros(q.shape)
    with np.errstate(invalid="ignore", over="ignore"):
        for i in range(n_q):
            j = np.flatnonzero(seen[i])
            if len(j) == 0:
                continue
            for h in range(H):
                s = scale * (k[j, h // g] @ q[i, h])
                m = np.nan if np.isnan(s).any() else s.max()
                p = np.exp(s - m)
                out[i, h] = (p @ v[j, h // g]) / p.sum()
    return out


def weights(logits, temperature):
    """Weights of a row's tokens, or None if it has no distribution."""
    x = np.array(logits, np.float64)
    x[np.isnan(x)] = -np.inf
    top = x.max()
    if top == -np.inf:
        return None
    if not temperature > 0:
        w = np.zeros(len(x))
        w[int(np.argmax(x == top))] = 1.0
        return w
    if top == np.inf:
        return (x == np.inf).astype(np.float64)
    w = np.zeros(len(x))
    some = x > -np.inf
    w[some] = np.exp((x[some] - top) / temperature)
    w[w < 2.0 ** -800] = 0.0  # (count as none)
    return w


def sample(w, u):
    """The first i whose running sum is above u times the whole; the last of a positive weight otherwise."""
    cum = np.cumsum(w)
    above = np.flatnonzero((cum > u * cum[-1]) & (w > 0))
    return int(above[0]) if len(above) else int(np.flatnonzero(w > 0)[-1])


def verify(parents, tokens, logits, temperature, u_sample, probs=None, u_accept=None):
    """(rows of the walk, next token) of one tree; parents None: a chain."""
    n = len(tokens)
    if n == 0:
        return [], -1
    parents = list(range(-1, n - 1)) if parents is None else list(parents)
    walk, cur = [0], 0
    while True:
        w = weights(logits[cur], temperature)
        if w is None:
            return walk, -1
        children = [i for i in range(cur + 1, n) if parents[i] == cur]
        if probs is None or not temperature > 0:
            token = sample(w, u_sample[cur] if temperature > 0 else 0.0)
            children = [i for i in children if tokens[i] == token]
            if not children:
                return walk, token
            cur = children[0]
        else:
            p = w / w.sum()
            q = np.where(probs[cur] > 0, probs[cur], 0.0).astype(np.float64)  # (NaN: 0)
            c, s, rest = 0.0, 1.0, p
            for i in children:
                x = tokens[i]
                if not 0 <= x < len(p):
                    continue
                if u_accept[i] * q[x] * s < rest[x]:
                    break
                c += s
                rest = np.maximum(p - c * q, 0.0)
                s = rest.sum()
            else:
                return walk, sample(rest if s > 0 else p, u_sample[cur])
            cur = i
        walk.append(cur)


def keep(rows, start, kept):
    """A sequence's rows with start + j replaced by what start + kept[j] was, as long as kept rises."""
    out, before = list(rows), -1
    for j, r in enumerate(kept):
        if not before < r < len(rows) - start:
            break
        out[start + j] = rows[start + r]
        before = r
    return out


def rotary(x, positions, freqs, axes, interleaved, index=None, inverse=False):
    """x [rows, heads, dim]; positions [axes, n]; returns float64."""
    x = np.array(x, np.float64)
    n = len(freqs)
    first, second = (slice(0, 2 * n, 2), slice(1, 2 * n, 2)) if interleaved else (slice(0, n), slice(n, 2 * n))
    for r in range(len(x)):
        t = r if index is None else int(index[r])
        if not 0 <= t < positions.shape[1]:
            continue
        # the product is exact in a long double's 64 bits or off by 2^-64 of itself
        a = [math.remainder(float(np.longdouble(f) * np.longdouble(int(positions[axes[i], t])) %
                                  (2 * np.longdouble("3.14159265358979323846264338327950288"))), 2 * math.pi)
             for i, f in enumerate(freqs)]
        z = (x[r][:, first] + 1j * x[r][:, second]) * np.exp((-1j if inverse else 1j) * np.array(a))
        x[r][:, first], x[r][:, second] = z.real, z.imag
    return x

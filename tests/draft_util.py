"""Helpers of drafted decoding's tests. Test infrastructure only."""
import numpy as np
import torch

from oracle import draft as od

DH = 128


def tree(rng, n, wide=0.7):
    """Parents of n rows: row 0 none, the others any row before (more of the early ones)."""
    return [-1] + [int(wide * i * rng.random()) for i in range(1, n)]


def up(x, dtype=None):
    t = torch.from_numpy(np.ascontiguousarray(x))
    return (t if dtype is None else t.to(dtype)).cuda()


def offsets(new):
    return np.concatenate([[0], np.cumsum(new)]).astype(np.int32)


def device_mask(seen, words, rows, junk=0):
    """Masks of a batch's sequences (seen: a matrix each), `rows` rows in all; `junk`: value of
    the rows behind the last and of bits behind a sequence's rows."""
    parts = []
    for s in seen:
        w = od.words(s, words)
        if junk:
            full = np.ones((s.shape[0], 32 * words), bool)
            full[:, :s.shape[1]] = s[:, :32 * words]
            w = od.words(full, words)
        parts.append(w)
    m = np.concatenate(parts + [np.full((rows - sum(len(p) for p in parts), words), junk, np.uint32)])
    return torch.from_numpy(m.view(np.int32)).cuda()


def attend(p, q, new, seen, words, scale=DH ** -0.5, cache=None, ws=True, stream=None, junk=0, mask=None, pad=3):
    """ce_paged_tree_attention on bf16 rows q; rows behind the last one are checked to stay as they were."""
    import paper_2608_29291_amd as ce
    c = cache or p.cache()
    qd = torch.from_numpy(q).to(torch.bfloat16).cuda()
    qd = torch.cat([qd, torch.zeros((pad,) + qd.shape[1:], dtype=torch.bfloat16, device="cuda")])
    o = torch.full(qd.shape, 77.0, dtype=torch.bfloat16, device="cuda")
    off, lens = up(offsets(new)), torch.tensor(p.lens, dtype=torch.int32).cuda()
    mask = device_mask(seen, words, len(qd), junk) if mask is None else mask
    w = ce.alloc_paged_workspace(c, qd.shape[0], qd.shape[1]) if ws else None
    if w is not None:
        w.fill_(0xff)  # NaN: what is on entry must not matter
    torch.cuda.synchronize()  # (the call may be made on another stream)
    ce.ce_paged_tree_attention(c, qd, o, off, lens, mask, scale, ws=w, stream=stream)
    torch.cuda.synchronize()
    o = o.float().cpu().numpy()
    assert (o[len(q):] == 77.0).all(), "rows behind the last were written"
    return o[:len(q)]


def visible(seen, n, m):
    """[n, m] truth values of a sequence of m keys, its n new ones last (some may not exist)."""
    out = np.ones((n, m), bool)
    for i in range(n):
        for j in range(m):
            k = j - (m - n)
            if k >= 0:
                out[i, j] = k < seen.shape[1] and seen[i, k]
    return out


def answer(p, q, new, seen, scale=DH ** -0.5):
    """float64 outputs and, per row and head, the largest value of the sequence."""
    out, top, at = np.zeros(q.shape), np.zeros(q.shape[:2]), 0
    g = q.shape[1] // p.hkv
    for b, n in enumerate(new):
        m = p.lens[b]
        out[at:at + n] = od.attend(q[at:at + n], p.k_used[b], p.v_used[b], visible(seen[b], n, m), scale)
        v = np.abs(np.where(np.isfinite(p.v_used[b]), p.v_used[b], 0.0))
        if len(v):
            top[at:at + n] = np.repeat(v.max((0, 2)), g)[None]
        at += n
    return out, top

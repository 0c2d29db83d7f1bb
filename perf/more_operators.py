"""Performance cases of drafted decoding over the paged key/value cache, and of rotary positions.

A step of a program that verifies a tree of drafted tokens: `ce_draft_masks` turns the
trees' parents into bits (who sees whom) and positions, `ce_paged_tree_attention` reads the
cache under them, `ce_verify_drafts` compares the drafts with the target's probabilities, and
`ce_kv_keep` with `ce_kv_trim` leave the accepted rows in the cache and give the other pages
back. `ce_rotary` turns queries and keys by their tokens' positions, in one axis or in several,
for drafted rows as for the packed rows of a prompt (which keep their tokens' positions).

Row 0 of a sequence is the last accepted token, rows 1 .. are the drafted ones, parents before
children. Lengths are written as text: `16*700` repeats, `551 8*1` is nine sequences.
"""
import math
import random

import torch

own = False

HEAD_DIM = 128
SCALE = 1.0 / math.sqrt(HEAD_DIM)
E4M3_MAX = 448.0

HEADS = [(12, 2), (28, 4), (4, 4), (8, 1)]
PAGES = [16, 32, 64, 128, 256]


def listed():
    return [
        # trees of a decoding step of 16 requests
        {"name": "masks_step", "op": "masks", "new": "16*26", "words": 1},
        # a full server with wide trees, and a few long chains
        {"name": "masks_server", "op": "masks", "new": "200*64 3*700 50*33 1 0 5", "words": 24},
        # one user's tree over a short cache: latency
        {"name": "tree_one", "op": "attend", "dtype": "bf16", "heads": 12, "kv_heads": 2, "page": 16, "new": "26",
         "lens": "1100", "what": "tree"},
        # a full server: trees of 64 over long 8-bit caches
        {"name": "tree_server_fp8", "op": "attend", "dtype": "e4m3", "heads": 28, "kv_heads": 4, "page": 64, "new": "24*64 8*33",
         "lens": "10*2100 10*4099 7*7001 5*16001", "what": "tree"},
        # chunks of two prompts: text is causal, the tokens of an image see all of it
        {"name": "image_chunks", "op": "attend", "dtype": "bf16", "heads": 28, "kv_heads": 4, "page": 32, "new": "1024 1001",
         "lens": "4300 1001", "what": "images"},
        # one user's tree against the target's probabilities: latency
        {"name": "verify_one", "op": "verify", "dtype": "bf16", "new": "9", "vocab": 65536, "draws": False, "temps": "one"},
        # trees of 16 requests over a large vocabulary, some of them greedy
        {"name": "verify_trees", "op": "verify", "dtype": "bf16", "new": "15*33 26", "vocab": 131072, "draws": False,
         "temps": "mixed"},
        # chains that a small model has drawn, with its probabilities, from a vocabulary of odd size
        {"name": "verify_chains", "op": "verify", "dtype": "f32", "new": "40*6 8*4", "vocab": 100003, "draws": True,
         "temps": "mixed"},
        # what is accepted of 16 trees, bf16 pages
        {"name": "keep_step", "op": "keep", "dtype": "bf16", "kv_heads": 4, "page": 16, "new": "16*33", "lens": "8*551 8*1001"},
        # and of a full server's, 8-bit pages
        {"name": "keep_server_fp8", "op": "keep", "dtype": "e4m3", "kv_heads": 4, "page": 64, "new": "200*64 56*17",
         "lens": "256*300"},
        # queries and keys of a drafted step, from the fused projection
        {"name": "rotary_step", "op": "rotary", "dtype": "bf16", "rows": 208, "heads": 32, "fused": 36, "dim": 128,
         "sections": "64", "interleaved": False, "packed": 0},
        # the retained rows of a denoising batch: time, height and width of their tokens
        {"name": "rotary_images", "op": "rotary", "dtype": "bf16", "rows": 17408, "heads": 32, "fused": 36, "dim": 128,
         "sections": "16 24 24", "interleaved": False, "packed": 21760},
    ]


# ---------------------------------------------------------------- drawn cases

def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _text(lens):
    return " ".join(map(str, lens))


def _draw_masks(rng):
    new = [rng.choice([rng.randint(1, 64), rng.randint(0, 64), _log_int(rng, 1, 700)]) for _ in range(_log_int(rng, 1, 256))]
    return {"op": "masks", "new": _text(new), "words": max(1, -(-max(new) // 32)) + rng.choice([0, 0, 1])}


def _draw_attend(rng):
    h, hkv = rng.choice(HEADS)
    what = rng.choice(["tree", "tree", "images"])
    if what == "tree":
        new = [rng.randint(1, 64) for _ in range(_log_int(rng, 1, 32))]
        lens = [n + _log_int(rng, 1, 16000) for n in new]
    else:
        new = [_log_int(rng, 2, 1024) for _ in range(rng.randint(1, 3))]
        lens = [n + rng.choice([0, _log_int(rng, 1, 4000)]) for n in new]
    return {"op": "attend", "dtype": rng.choice(["bf16", "e4m3"]), "heads": h, "kv_heads": hkv, "page": rng.choice(PAGES),
            "new": _text(new), "lens": _text(lens), "what": what}


def _draw_verify(rng):
    draws = rng.random() < 0.4
    new = [rng.randint(1, 8 if draws else 40) for _ in range(_log_int(rng, 1, 64))]
    return {"op": "verify", "dtype": rng.choice(["bf16", "f32"]), "new": _text(new), "vocab": _log_int(rng, 1000, 160000),
            "draws": draws, "temps": rng.choice(["one", "mixed"])}


def _draw_keep(rng):
    _, hkv = rng.choice(HEADS)
    new = [rng.randint(0, 64) for _ in range(_log_int(rng, 1, 256))]
    return {"op": "keep", "dtype": rng.choice(["bf16", "e4m3"]), "kv_heads": hkv, "page": rng.choice(PAGES), "new": _text(new),
            "lens": _text([n + rng.randint(0, 400) for n in new])}


def _draw_rotary(rng):
    dim = rng.choice([64, 72, 80, 96, 128, 128, 128, 256])
    half = dim // 2
    a = rng.randint(1, half - 2)
    b = rng.randint(1, half - a - 1)
    sections = rng.choice([[half], [half], [a, half - a], [a, b, half - a - b]])
    rows, heads = _log_int(rng, 1, 17408), rng.randint(1, 32)
    return {"op": "rotary", "dtype": rng.choice(["bf16", "f32"]), "rows": rows, "heads": heads,
            "fused": heads + rng.choice([0, 2, 8]), "dim": dim, "sections": _text(sections),
            "interleaved": rng.random() < 0.4, "packed": rng.choice([0, rows + rng.randint(0, rows)])}


def draw(rng):
    makers = {"masks": _draw_masks, "attend": _draw_attend, "verify": _draw_verify, "keep": _draw_keep, "rotary": _draw_rotary}
    op = rng.choice(["masks", "attend", "attend", "verify", "verify", "keep", "rotary", "rotary"])
    same = [c for c in listed() if c["op"] == op]
    most = {k: max(work(c)[k] for c in same) for k in ("flops", "bytes")}
    most_padded = max(_padded(c) for c in same)
    while True:
        c = makers[op](rng)
        w = work(c)
        if "new" in c and not any(_ints(c["new"])):
            continue
        if w["flops"] <= most["flops"] and w["bytes"] <= most["bytes"] and _padded(c) <= most_padded:
            return c


# -------------------------------------------------------------- case helpers

def _ints(text):
    out = []
    for part in text.split():
        n, _, x = part.rpartition("*")
        out += [int(x)] * (int(n) if n else 1)
    return out


def _ceil(a, b):
    return -(-a // b)


def _padded(case):
    """Scores that the plain form of an attention holds (it pads to the longest)."""
    if case["op"] != "attend":
        return 0
    new, lens = _ints(case["new"]), _ints(case["lens"])
    return len(new) * case["heads"] * max(new) * (max(lens) + case["page"])


def _tree(n, b, chain=False):
    """Parents of a sequence's n rows (b: its number): the shape belongs to the case."""
    rng = random.Random(1009 * n + b)
    return [-1 if i == 0 else i - 1 if chain else int(0.7 * i * rng.random()) for i in range(n)]


def _trees(case):
    """(A long row of drafts is a chain.)"""
    chains = case["op"] == "verify" and case["draws"]
    return [_tree(n, b, chains or n > 64) for b, n in enumerate(_ints(case["new"]))]


def _depths(parents):
    out = []
    for p in parents:
        out.append(0 if p < 0 else out[p] + 1)
    return out


def _segments(n, b):
    """Ends of a prompt's segments, text and image in turn."""
    rng = random.Random(7919 * n + b)
    out = []
    while not out or out[-1] < n:
        out.append(min(n, (out[-1] if out else 0) + (rng.randint(1, 120) if len(out) % 2 == 0 else rng.randint(64, 400))))
    return out


def _seen(case, b, n):
    """[n, n] truth values: which of a sequence's new rows see which."""
    seen = torch.zeros((n, n), dtype=torch.bool)
    if case["what"] == "tree":
        for i, p in enumerate(_tree(n, b, n > 64)):
            if p >= 0:
                seen[i] = seen[p]
            seen[i, i] = True
        return seen
    seen = torch.ones((n, n), dtype=torch.bool).tril()
    ends = _segments(n, b)
    for k in range(1, len(ends), 2):
        seen[ends[k - 1]:ends[k], ends[k - 1]:ends[k]] = True
    return seen


def _words(case):
    return max(1, _ceil(max(_ints(case["new"])), 32))


def _pack(seen, words):
    """Truth values [n, n] as 32-bit words [n, words]: bit j % 32 of word j / 32."""
    n = seen.shape[0]
    bits = torch.zeros((n, words * 32), dtype=torch.int64)
    bits[:, :n] = seen
    x = (bits.view(n, words, 32) << torch.arange(32)).sum(-1)
    return torch.where(x >= 1 << 31, x - (1 << 32), x).to(torch.int32)


def _width(case):
    return {"e4m3": 1, "bf16": 2, "f32": 4}[case["dtype"]]


def _kept(case):
    """Rows that are accepted of every sequence. (Rows below the count stay where they are,
    others come from behind it, so that a pass finds what the one before it found.)"""
    out = []
    for b, n in enumerate(_ints(case["new"])):
        rng = random.Random(31 * n + b)
        m = min(n, rng.randint(1, 7))
        moved = rng.randint(0, m - 1) if n else 0
        moved = min(moved, n - m)
        out.append(list(range(m - moved)) + sorted(rng.sample(range(m, n), moved)))
    return out


def work(case):
    op = case["op"]
    if op == "rotary":
        pairs = case["rows"] * case["heads"] * (case["dim"] // 2)
        axes = len(_ints(case["sections"]))
        return {"bytes": 4 * pairs * _width(case) + 4 * axes * case["rows"] + (4 * case["rows"] if case["packed"] else 0),
                "flops": 6 * pairs}
    new = _ints(case["new"])
    rows = sum(new)
    if op == "masks":
        return {"bytes": 4 * (2 * len(new) + 1) + rows * (8 + 4 * case["words"]), "flops": 0}
    if op == "verify":
        # all logits, of the drafts' probabilities the row where a sequence ends
        return {"bytes": rows * (case["vocab"] * _width(case) + 16) + (len(new) * case["vocab"] * 4 if case["draws"] else 0),
                "flops": rows * case["vocab"] * 3}
    if op == "keep":
        moved = sum(sum(r != j for j, r in enumerate(k)) for k in _kept(case))
        before = _ints(case["lens"])
        page = case["page"]
        back = sum(_ceil(m, page) - _ceil(m - n + len(k), page) for m, n, k in zip(before, new, _kept(case)))
        return {"bytes": moved * 4 * case["kv_heads"] * HEAD_DIM * _width(case) + 4 * sum(map(len, _kept(case))) +
                20 * len(new) + 8 * back, "flops": 0}
    keys = sum(_ints(case["lens"]))
    pairs = sum(n * (m - n) + int(_seen(case, b, n).sum()) for b, (n, m) in enumerate(zip(new, _ints(case["lens"]))))
    return {"bytes": 2 * rows * case["heads"] * HEAD_DIM * 2 + keys * (2 * case["kv_heads"] * HEAD_DIM * _width(case)) +
            4 * rows * _words(case), "flops": 4 * HEAD_DIM * case["heads"] * pairs}


# -------------------------------------------------------------------- inputs

def _dev(x, dtype=torch.int32):
    return torch.tensor(x, dtype=dtype).cuda()


def _offsets(new):
    out = [0]
    for n in new:
        out.append(out[-1] + n)
    return out


def _table(gen, lens, page, spare, width):
    """Pages in the order that a long-running pool has them: any; the rest is free."""
    held = [_ceil(m, page) for m in lens]
    n_pages = sum(held) + spare
    order = torch.randperm(n_pages, generator=gen, dtype=torch.int64).to(torch.int32)
    table = torch.full((len(lens), width), -1, dtype=torch.int32)
    at = 0
    for b, n in enumerate(held):
        table[b, :n] = order[at:at + n]
        at += n
    return table.cuda(), order, at, n_pages


def _pages(case, n_pages, gen):
    """Keys and values of the whole pool with the scales of an 8-bit one."""
    shape = (n_pages, case["kv_heads"], case["page"], HEAD_DIM)
    k = torch.randn(shape, dtype=torch.bfloat16, device="cuda", generator=gen)
    v = torch.randn(shape, dtype=torch.bfloat16, device="cuda", generator=gen)
    if case["dtype"] == "bf16":
        return k, v, None, None
    # |x| <= about 5.5 for normal values: the largest lands near the top of e4m3
    ks = torch.rand(case["kv_heads"], device="cuda", generator=gen) * 0.01 + 0.012
    vs = torch.rand(case["kv_heads"], device="cuda", generator=gen) * 0.01 + 0.012
    return _quantize(k, ks[:, None, None]), _quantize(v, vs[:, None, None]), ks, vs


def _quantize(x, scale):
    return (x.float() / scale).clamp(-E4M3_MAX, E4M3_MAX).to(torch.float8_e4m3fn)


def _freqs(case, base=10000.0):
    """Radians a position of every pair, and the axis that it turns by."""
    half = case["dim"] // 2
    axes = [a for a, n in enumerate(_ints(case["sections"])) for _ in range(n)]
    return [base ** (-i / half) for i in range(half)], axes


def prepare(case, seed):
    cpu = torch.Generator().manual_seed(seed)
    gen = torch.Generator(device="cuda").manual_seed(seed)
    s = {"case": case}
    op = case["op"]
    {"masks": _prepare_masks, "attend": _prepare_attend, "verify": _prepare_verify, "keep": _prepare_keep,
     "rotary": _prepare_rotary}[op](s, case, cpu, gen)
    return s


def _prepare_masks(s, case, cpu, gen):
    new = _ints(case["new"])
    rows, trees = sum(new), _trees(case)
    s.update(offsets=_dev(_offsets(new)), parents=_dev([p for t in trees for p in t]),
             base=torch.randint(0, 20000, (len(new),), generator=cpu).to(torch.int32).cuda(),
             depth=max((max(_depths(t)) for t in trees if t), default=0),
             mask=torch.zeros((rows, case["words"]), dtype=torch.int32, device="cuda"),
             positions=torch.zeros(rows, dtype=torch.int32, device="cuda"))
    if own:
        import paper_2608_29291_amd as ce
        s["drafts"] = ce.Drafts(s["offsets"], s["parents"])


def _prepare_attend(s, case, cpu, gen):
    new, lens, page = _ints(case["new"]), _ints(case["lens"]), case["page"]
    words = _words(case)
    s["table"], _, _, n_pages = _table(cpu, lens, page, 3, max(_ceil(m, page) for m in lens) + 1)
    s["k"], s["v"], s["ks"], s["vs"] = _pages(case, n_pages, gen)
    s["q"] = torch.randn((sum(new), case["heads"], HEAD_DIM), dtype=torch.bfloat16, device="cuda", generator=gen)
    s["o"] = torch.empty_like(s["q"])
    s["mask"] = torch.cat([_pack(_seen(case, b, n), words) for b, n in enumerate(new)]).cuda()
    s.update(offsets=_dev(_offsets(new)), lens=_dev(lens), most=max(new), most_keys=max(lens))
    if own:
        import paper_2608_29291_amd as ce
        s["cache"] = ce.KVCache(s["k"], s["v"], s["table"], s["ks"], s["vs"])
        s["ws"] = ce.alloc_paged_workspace(s["cache"], s["q"].shape[0], case["heads"])


def _prepare_verify(s, case, cpu, gen):
    new, vocab = _ints(case["new"]), case["vocab"]
    rows, trees = sum(new), _trees(case)
    parents = torch.tensor([p for t in trees for p in t], dtype=torch.int32).cuda()
    dtype = torch.bfloat16 if case["dtype"] == "bf16" else torch.float32
    logits = torch.randn((rows, vocab), device="cuda", generator=gen) * 2.0
    off = torch.tensor(_offsets(new)[:-1], device="cuda")
    b = torch.repeat_interleave(torch.arange(len(new), device="cuda"), torch.tensor(new, device="cuda"))
    up = torch.where(parents >= 0, off[b] + parents, -1)  # the parent's row of the batch
    child = torch.nonzero(up >= 0).flatten()
    tokens = torch.randint(0, vocab, (rows,), device="cuda", generator=gen)
    probs = None
    if case["draws"]:  # the small model's distribution, and tokens drawn from it
        probs = torch.softmax(logits + 0.5 * torch.randn((rows, vocab), device="cuda", generator=gen) +
                              6.0 * (torch.rand((rows, vocab), device="cuda", generator=gen) > 0.9999), -1)
        logits += 6.0 * (probs > 100.0 / vocab) * (probs > 2e-3)
        tokens[child] = torch.multinomial(probs[up[child]], 1, generator=gen).flatten()
    else:  # drafts are likely tokens
        top = math.log(vocab) + 2.0 + torch.randn(child.numel(), device="cuda", generator=gen)
        logits[up[child], tokens[child]] = top
    temps = torch.ones(len(new), device="cuda")
    if case["temps"] == "mixed":
        temps = 0.5 + 0.7 * torch.rand(len(new), device="cuda", generator=gen)
        temps[::3] = 0.0
    s.update(offsets=_dev(_offsets(new)), parents=parents, tokens=tokens.to(torch.int32), logits=logits.to(dtype), probs=probs,
             temps=temps, u_accept=torch.rand(rows, device="cuda", generator=gen),
             u_sample=torch.rand(rows, device="cuda", generator=gen), most=max(new),
             kept=torch.full((rows,), -1, dtype=torch.int32, device="cuda"), n_kept=_dev([0] * len(new)),
             next=_dev([0] * len(new)))
    if own:
        import paper_2608_29291_amd as ce
        s["drafts"] = ce.Drafts(s["offsets"], s["parents"], s["tokens"])
        s["ws"] = ce.alloc_verify_workspace(s["drafts"], vocab)


def _prepare_keep(s, case, cpu, gen):
    new, lens, page = _ints(case["new"]), _ints(case["lens"]), case["page"]
    kept = _kept(case)
    table, order, at, n_pages = _table(cpu, lens, page, 40, max(_ceil(m, page) for m in lens) + 1)
    free = torch.zeros(n_pages, dtype=torch.int32)
    free[:n_pages - at] = order[at:]
    s["k"], s["v"], s["ks"], s["vs"] = _pages(case, n_pages, gen)
    s.update(table=table, lens=_dev(lens), offsets=_dev(_offsets(new)), start=_dev([m - n for m, n in zip(lens, new)]),
             kept=_dev([r for n, k in zip(new, kept) for r in k + [-1] * (n - len(k))]), n_kept=_dev([len(k) for k in kept]),
             free=free.cuda(), count=_dev([n_pages - at]), lens_out=_dev([0] * len(new)), count_out=_dev([0]))
    if own:
        import paper_2608_29291_amd as ce
        s["cache"] = ce.KVCache(s["k"], s["v"], s["table"], s["ks"], s["vs"])


def _prepare_rotary(s, case, cpu, gen):
    rows, heads, dim = case["rows"], case["heads"], case["dim"]
    dtype = torch.bfloat16 if case["dtype"] == "bf16" else torch.float32
    n = case["packed"] or rows
    axes = len(_ints(case["sections"]))
    fused = torch.randn((rows, case["fused"], dim), dtype=dtype, device="cuda", generator=gen)
    pos = torch.randint(0, 30000, (1, n), generator=cpu) + (torch.randint(0, 64, (axes, n), generator=cpu) if axes > 1 else 0)
    s.update(x=fused[:, :heads], y=torch.empty((rows, heads, dim), dtype=dtype, device="cuda"),
             positions=pos.to(torch.int32).cuda(), index=None)
    if case["packed"]:  # the retained tokens of the batch, in order
        s["index"] = torch.randperm(n, generator=cpu)[:rows].sort()[0].to(torch.int32).cuda()
    freqs, of = _freqs(case)
    s["freqs"], s["of"] = torch.tensor(freqs, dtype=torch.float64).cuda(), torch.tensor(of).cuda()
    if own:
        import paper_2608_29291_amd as ce
        s["rotary"] = ce.Rotary(freqs, of, interleaved=case["interleaved"])


# ----------------------------------------------------------------- one pass

def run(s):
    return {"masks": _masks, "attend": _attend, "verify": _verify, "keep": _keep, "rotary": _rotary}[s["case"]["op"]](s)


def _rows_of(s, n):
    """Sequence of each row, and its row 0."""
    off = s["offsets"].long()
    b = torch.searchsorted(off[1:].contiguous(), torch.arange(n, device=off.device), right=True)
    return b, off[b]


def _masks(s):
    if own:
        import paper_2608_29291_amd as ce
        ce.ce_draft_masks(s["drafts"], s["mask"], positions=s["positions"], base=s["base"])
        return {"mask": s["mask"], "positions": s["positions"]}
    words = s["case"]["words"]
    n = s["parents"].numel()
    b, first = _rows_of(s, n)
    parents = s["parents"].long()
    rows = torch.arange(n + 1, device=parents.device)
    # row n stands for no parent and sees nobody; the reach of a row doubles each time
    up = torch.cat([torch.where(parents >= 0, first + parents, n), parents.new_full((1,), n)])
    bits = torch.zeros((n + 1, 32 * words), dtype=torch.bool, device=parents.device)
    bits[rows[:n], rows[:n] - first] = True
    reach = 1
    while reach <= s["depth"]:
        bits, up, reach = bits | bits[up], up[up], 2 * reach
    bits = bits[:n]
    depth = bits.sum(-1) - 1
    x = (bits.reshape(n, words, 32).long() << torch.arange(32, device=parents.device)).sum(-1)
    return {"mask": torch.where(x >= 1 << 31, x - (1 << 32), x).to(torch.int32),
            "positions": (s["base"].long()[b] + depth).to(torch.int32)}


def _attend(s):
    c = s["case"]
    if own:
        import paper_2608_29291_amd as ce
        ce.ce_paged_tree_attention(s["cache"], s["q"], s["o"], s["offsets"], s["lens"], s["mask"], SCALE, ws=s["ws"])
        return s["o"]
    h, hkv, page = c["heads"], c["kv_heads"], c["page"]
    b, width, g = s["lens"].numel(), _ceil(s["most_keys"], page), h // hkv
    pages = s["table"][:, :width].clamp(min=0).flatten().long()

    def rows(pool, scale):  # [B, H_kv, keys, 128]
        x = pool[pages] if scale is None else pool.view(torch.uint8)[pages].view(pool.dtype)
        x = x.float() if scale is None else x.float() * scale[:, None, None]
        return x.view(b, width, hkv, page, HEAD_DIM).transpose(1, 2).reshape(b, hkv, width * page, HEAD_DIM)

    off, lens = s["offsets"].long(), s["lens"].long()
    n = off[1:] - off[:-1]
    i, j = torch.arange(s["most"], device=off.device), torch.arange(width * page, device=off.device)
    at = (off[:-1, None] + i).clamp(max=off[-1] - 1)
    q = s["q"][at].float().view(b, s["most"], hkv, g, HEAD_DIM).permute(0, 2, 3, 1, 4).reshape(b, hkv, -1, HEAD_DIM)
    score = torch.matmul(q, rows(s["k"], s["ks"]).transpose(2, 3)).view(b, hkv, g, s["most"], -1).mul_(SCALE)
    # new key j of a sequence is bit j of a row's words
    new = (j - (lens - n)[:, None])[:, None]  # [B, 1, keys]
    word = (new >> 5).clamp(0, s["mask"].shape[1] - 1).expand(b, s["most"], -1)
    bit = (torch.gather(s["mask"].long()[at], 2, word) >> (new & 31)) & 1
    seen = (j < lens[:, None])[:, None] & ((new < 0) | (bit != 0))  # [B, queries, keys]
    score.masked_fill_(~seen[:, None, None], -math.inf)
    top = score.amax(-1, keepdim=True)
    any_seen = seen.any(-1)[:, None, None, :, None]
    score.sub_(torch.where(any_seen, top, 0.0)).exp_()
    total = score.sum(-1, keepdim=True)
    out = torch.matmul(score.view(b, hkv, -1, width * page), rows(s["v"], s["vs"])).view(b, hkv, g, s["most"], HEAD_DIM)
    out = torch.where(any_seen, out / total, 0.0)
    out = out.permute(0, 3, 1, 2, 4).reshape(b * s["most"], h, HEAD_DIM).to(s["q"].dtype)
    # row r of the batch is row r - off[b] of its sequence b
    r = torch.arange(s["q"].shape[0], device=off.device)
    seq, first = _rows_of(s, r.numel())
    return out[seq * s["most"] + r - first]


def _weights(logits, temps):
    """Weights of a row's tokens, the largest 1, in 64 bits (sums of 1e5 of them have borders
    1e-5 apart); temperature 0: the lowest of the largest."""
    x = logits.double()
    top = x.amax(-1, keepdim=True)
    index = torch.arange(x.shape[1], device=x.device)
    lowest = torch.where(x == top, index, x.shape[1]).amin(-1, keepdim=True)
    hot = temps[:, None] > 0
    w = torch.exp((x - top) / torch.where(hot, temps[:, None].double(), 1.0))
    return torch.where(hot, w, (index == lowest).double())


def _pick(w, u):
    """The first index whose running sum is above u times the whole."""
    cum = torch.cumsum(w, -1)
    return (cum <= u.double()[:, None] * cum[:, -1:]).sum(-1).clamp(max=w.shape[1] - 1)


def _verify(s):
    if own:
        import paper_2608_29291_amd as ce
        ce.ce_verify_drafts(s["drafts"], s["logits"], s["u_sample"], s["kept"], s["n_kept"], s["next"], temperature=s["temps"],
                            draft_probs=s["probs"], u_accept=s["u_accept"] if s["probs"] is not None else None, ws=s["ws"])
        return {"kept": s["kept"], "n_kept": s["n_kept"], "next": s["next"]}
    n = s["parents"].numel()
    b, first = _rows_of(s, n)
    rows = torch.arange(n, device=b.device)
    tokens, parents = s["tokens"].long(), s["parents"].long()
    up = torch.where(parents >= 0, first + parents, n)
    w = _weights(s["logits"], s["temps"][b])
    if s["probs"] is None:
        picked = torch.cat([_pick(w, s["u_sample"]), b.new_full((1,), -1)])
        good = tokens == picked[up]
        # of equal siblings the first
        key = up * s["case"]["vocab"] + tokens
        lowest = rows.new_full((n,), n).scatter_reduce(0, torch.unique(key, return_inverse=True)[1], rows, "amin")
        good &= lowest[torch.unique(key, return_inverse=True)[1]] == rows
    else:  # chains: accepted with probability p / q
        p = w / w.sum(-1, keepdim=True)
        before = up.clamp(max=n - 1)
        good = (s["u_accept"].double() * s["probs"][before, tokens].double() < p[before, tokens]) & (up < n)
    good = torch.cat([good | (rows == first), good.new_zeros(1)])  # row 0 is accepted as it is
    for _ in range(s["most"]):
        good = torch.cat([good[:-1] & ((rows == first) | good[up]), good.new_zeros(1)])
    good = good[:-1]
    # the accepted rows, in order, then -1
    rank = torch.cumsum(good, 0) - good.long()
    place = first + rank - rank[first]
    kept = torch.cat([rows.new_full((n,), -1), rows.new_zeros(1)])
    kept = kept.scatter(0, torch.where(good, place, n), rows - first)[:n]
    n_kept = torch.zeros_like(s["n_kept"], dtype=torch.int64).index_add(0, b, good.long())
    off = s["offsets"].long()
    have = off[1:] > off[:-1]
    last = (off[:-1] + kept[(off[:-1] + n_kept - 1).clamp(0, n - 1)].clamp(min=0)).clamp(max=n - 1)
    if s["probs"] is None:
        token = picked[last]
    else:  # a chain that ends before its last row ends with a rejection
        rest = p[last]
        short = ((last + 1 < off[1:]) & (s["temps"] > 0))[:, None]
        rest = torch.where(short, (rest - s["probs"][last].double()).clamp(min=0.0), rest)
        token = _pick(rest, s["u_sample"][last])
    i32 = torch.int32
    return {"kept": kept.to(i32), "n_kept": n_kept.to(i32), "next": torch.where(have, token, -1).to(i32)}


def _keep(s):
    if own:
        import paper_2608_29291_amd as ce
        ce.ce_kv_keep(s["cache"], s["offsets"], s["start"], s["kept"], s["n_kept"])
        ce.ce_kv_trim(s["cache"], s["lens"], s["start"], s["n_kept"], s["free"], s["count"], lens_out=s["lens_out"],
                      free_count_out=s["count_out"])
        return {"k": s["k"], "v": s["v"], "free": s["free"], "count": s["count_out"], "lens": s["lens_out"]}
    page, table = s["case"]["page"], s["table"]
    n = s["kept"].numel()
    b, first = _rows_of(s, n)
    j = torch.arange(n, device=b.device) - first
    start, n_kept = s["start"].long(), s["n_kept"].long()
    to = start[b] + j
    of = start[b] + torch.where(j < n_kept[b], s["kept"].long(), j)

    def place(token):
        return table[b, token // page].long(), token % page

    (p0, r0), (p1, r1) = place(of), place(to)
    for pool in (s["k"], s["v"]):
        pool = pool if s["ks"] is None else pool.view(torch.uint8)
        pool[p1, :, r1] = pool[p0, :, r0]
    lens = start + n_kept
    held, need = (s["lens"].long() + page - 1) // page, (lens + page - 1) // page
    back = held - need
    at = s["count"].long() + torch.cumsum(back, 0) - back
    col = torch.arange(table.shape[1], device=b.device)
    mine = (col >= need[:, None]) & (col < held[:, None])
    to = torch.where(mine, at[:, None] + col - need[:, None], s["free"].numel())
    free = torch.cat([s["free"], s["free"].new_zeros(1)]).scatter(0, to.flatten(), table.flatten())[:-1]
    return {"k": s["k"], "v": s["v"], "free": free, "count": (s["count"].long() + back.sum()).to(torch.int32),
            "lens": lens.to(torch.int32)}


def _halves(x, interleaved):
    return (x[..., ::2], x[..., 1::2]) if interleaved else (x[..., :x.shape[-1] // 2], x[..., x.shape[-1] // 2:])


def _rotary(s):
    if own:
        import paper_2608_29291_amd as ce
        ce.ce_rotary(s["rotary"], s["x"], s["y"], s["positions"], index=s["index"])
        return s["y"]
    return _turn(s, torch.float32).to(s["x"].dtype)


def _turn(s, dtype):
    pos = s["positions"] if s["index"] is None else s["positions"][:, s["index"].long()]
    angle = pos.double()[s["of"]].t() * s["freqs"]  # [rows, pairs]: far positions need 64 bits
    cos, sin = angle.cos().to(dtype)[:, None], angle.sin().to(dtype)[:, None]
    inter = s["case"]["interleaved"]
    a, b = _halves(s["x"].to(dtype), inter)
    pair = [a * cos - b * sin, a * sin + b * cos]
    return torch.stack(pair, -1).flatten(2) if inter else torch.cat(pair, -1)


# ------------------------------------------------------- the definition, 64 bits

def exact(case, seed):
    if case["op"] in ("masks", "verify"):
        return None  # whole numbers
    s = prepare(case, seed)
    if case["op"] == "rotary":
        z = torch.view_as_complex(torch.stack(_halves(s["x"].double(), case["interleaved"]), -1).contiguous())
        pos = s["positions"].double()
        if s["index"] is not None:
            pos = pos[:, s["index"].long()]
        phase = torch.polar(torch.ones((), dtype=torch.float64, device="cuda"), pos[s["of"]].t() * s["freqs"])
        out = torch.view_as_real(z * phase[:, None])
        return out.flatten(2) if case["interleaved"] else torch.cat([out[..., 0], out[..., 1]], -1)
    new, lens, page = _ints(case["new"]), _ints(case["lens"]), case["page"]
    if case["op"] == "keep":  # values are moved as they are
        k, v, at = s["k"].double(), s["v"].double(), 0
        for b, (n, m, rows) in enumerate(zip(new, lens, _kept(case))):
            to = torch.arange(len(rows), device="cuda") + m - n
            of = torch.tensor(rows, dtype=torch.int64, device="cuda") + m - n
            for pool in (k, v):
                ids = s["table"][b].long()
                pool[ids[to // page], :, to % page] = pool[ids[of // page], :, of % page]
        return {"k": k, "v": v, "free": None, "count": None, "lens": None}
    h, hkv = case["heads"], case["kv_heads"]
    g = h // hkv
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    at = 0
    for b, (n, m) in enumerate(zip(new, lens)):
        ids = s["table"][b, :_ceil(m, page)].long()
        hide = ~_seen(case, b, n).cuda()
        for kh in range(hkv):
            kv = []
            for pool, scale in ((s["k"], s["ks"]), (s["v"], s["vs"])):
                x = (pool if scale is None else pool.view(torch.uint8))[ids, kh]
                x = x.double() if scale is None else x.view(pool.dtype).double() * scale[kh].double()
                kv.append(x.reshape(-1, HEAD_DIM)[:m].contiguous())
            for hq in range(kh * g, (kh + 1) * g):
                x = torch.matmul(s["q"][at:at + n, hq].double(), kv[0].t().contiguous()) / math.sqrt(HEAD_DIM)
                x[:, m - n:].masked_fill_(hide, -math.inf)
                out[at:at + n, hq] = torch.matmul(torch.softmax(x, -1), kv[1])
        at += n
    return out

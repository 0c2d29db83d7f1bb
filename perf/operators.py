"""Performance cases of the paged key/value cache: page tables, writes, attention.

Three operators that a serving program calls per layer and step, in this order:
`ce_kv_reserve` gives the new rows of every sequence pages and slots on the
device (the packed row counts of a routed layer are known only there),
`ce_kv_append` writes their keys and values into the pages, `ce_paged_attention`
reads the cache. Pages are [n_pages, kv_heads, page, 128] in bf16 or e4m3 (with
a scale per head); tables, lists and lengths are int32.

Lengths are written as text: `16*700` repeats, `551 8*1` is nine sequences.
"""
import math

import torch

own = False

HEAD_DIM = 128
SCALE = 1.0 / math.sqrt(HEAD_DIM)
E4M3_MAX = 448.0

HEADS = [(12, 2), (28, 4), (4, 4), (8, 1)]
PAGES = [16, 32, 64, 128, 256]


def listed():
    return [
        # a decoding step of 64 running requests: one slot each, now and then a page
        {"name": "reserve_decode", "op": "reserve", "page": 16, "new": "64*1",
         "lens": "9*666 7*1021 551 15*1895 12*2437 5*3100 15*160", "ended": 0, "spare": 64},
        # a large mixed step: prompts packed by a routed layer beside decodes, some
        # places in the batch handed from ended requests to new ones
        {"name": "reserve_prefill", "op": "reserve", "page": 16, "new": "8*551 4*2176 100*1 5*700 120*1 19*0",
         "lens": "12*900 100*2000 5*1300 120*777 19*431", "ended": 31, "spare": 2000},
        # the same decoding step's keys and values, as the projection leaves them
        {"name": "append_decode", "op": "append", "dtype": "bf16", "kv_heads": 4, "page": 16, "rows": 64, "pad": 0,
         "fused": 28},
        # a denoising batch's retained rows into an 8-bit cache, from a fused projection
        # sized for more rows than were kept
        {"name": "append_prefill_fp8", "op": "append", "dtype": "e4m3", "kv_heads": 4, "page": 64, "rows": 17408,
         "pad": 300, "fused": 28},
        # a decoding step over compressed caches of many lengths
        {"name": "attend_decode", "op": "attend", "dtype": "bf16", "heads": 28, "kv_heads": 4, "page": 16, "new": "16*1",
         "lens": "4*666 3*1021 551 5*1895 2*2437 3100", "causal": True},
        # a full server: many requests with long contexts in 8 bits
        {"name": "attend_decode_fp8", "op": "attend", "dtype": "e4m3", "heads": 28, "kv_heads": 4, "page": 64,
         "new": "64*1", "lens": "20*2100 16*4099 12*7001 10*9000 6*16001", "causal": True},
        # one user with a very long context
        {"name": "attend_one_long", "op": "attend", "dtype": "bf16", "heads": 28, "kv_heads": 4, "page": 32, "new": "1",
         "lens": "65537", "causal": True},
        # drafted tokens of a few requests verified together
        {"name": "attend_drafts", "op": "attend", "dtype": "bf16", "heads": 12, "kv_heads": 2, "page": 16, "new": "8*5",
         "lens": "1029 2*2051 333 4*4103", "causal": True},
        # one chunk of a long prompt over what is cached of it
        {"name": "attend_chunk", "op": "attend", "dtype": "bf16", "heads": 28, "kv_heads": 4, "page": 16, "new": "512",
         "lens": "8704", "causal": True},
        # chunks of two prompts beside thirty decodes, 8-bit cache
        {"name": "attend_mixed_fp8", "op": "attend", "dtype": "e4m3", "heads": 12, "kv_heads": 2, "page": 32,
         "new": "2*701 30*1", "lens": "701 2900 10*500 12*1500 8*2811", "causal": True},
        # a denoising step: retained latents see the prompt and each other
        {"name": "attend_generation", "op": "attend", "dtype": "bf16", "heads": 12, "kv_heads": 2, "page": 64,
         "new": "4*2176", "lens": "4*2304", "causal": False},
        # the largest step: chunks of four long prompts at the 7B heads
        {"name": "attend_chunks_long", "op": "attend", "dtype": "bf16", "heads": 28, "kv_heads": 4, "page": 64,
         "new": "4*2048", "lens": "2*10240 7000 9001", "causal": True},
    ]


# ---------------------------------------------------------------- drawn cases

def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _text(lens):
    return " ".join(map(str, lens))


def _draw_reserve(rng):
    b = _log_int(rng, 1, 600)
    new = [rng.choice([1, 1, 1, 1, 0, _log_int(rng, 1, 3000)]) if i >= 16 or rng.random() < 0.5 else _log_int(rng, 1, 3000)
           for i in range(b)]
    return {"op": "reserve", "page": rng.choice(PAGES), "new": _text(new), "lens": _text([_log_int(rng, 1, 4000) for _ in new]),
            "ended": rng.randint(0, b // 2), "spare": _log_int(rng, 1, 4000)}


def _draw_append(rng):
    h, hkv = rng.choice(HEADS)
    return {"op": "append", "dtype": rng.choice(["bf16", "e4m3"]), "kv_heads": hkv, "page": rng.choice(PAGES),
            "rows": _log_int(rng, 1, 17408), "pad": rng.choice([0, 0, rng.randint(1, 500)]), "fused": rng.choice([0, h])}


def _draw_attend(rng):
    h, hkv = rng.choice(HEADS)
    what = rng.choice(["decode", "drafts", "chunk", "prefill", "mixed", "generation"])
    if what == "decode":
        new = [1] * _log_int(rng, 1, 64)
        lens = [_log_int(rng, 1, 16384) for _ in new]
    elif what == "drafts":
        new = [rng.randint(2, 9) for _ in range(_log_int(rng, 1, 32))]
        lens = [n + _log_int(rng, 1, 8192) for n in new]
    elif what == "mixed":
        new = [_log_int(rng, 10, 1000) for _ in range(rng.randint(1, 3))] + [1] * rng.randint(1, 24)
        lens = [n + _log_int(rng, 1, 4000) for n in new]
    else:
        new = [_log_int(rng, 16, 2048) for _ in range(rng.randint(1, 4))]
        lens = [n + (0 if what == "prefill" else _log_int(rng, 1, 8192)) for n in new]
    return {"op": "attend", "dtype": rng.choice(["bf16", "e4m3"]), "heads": h, "kv_heads": hkv, "page": rng.choice(PAGES),
            "new": _text(new), "lens": _text(lens), "causal": what != "generation"}


def draw(rng):
    most = {k: max(work(c)[k] for c in listed()) for k in ("flops", "bytes")}
    while True:
        c = rng.choice([_draw_reserve, _draw_append, _draw_attend, _draw_attend, _draw_attend, _draw_attend])(rng)
        w = work(c)
        if w["flops"] <= most["flops"] and w["bytes"] <= most["bytes"] and _padded(c) <= _padded(listed()[-1]):
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


def _visible(case):
    """Query/key pairs of one head, and the keys that some query sees."""
    pairs = keys = 0
    for n, m in zip(_ints(case["new"]), _ints(case["lens"])):
        if not case["causal"]:
            pairs, keys = pairs + n * m, keys + (m if n else 0)
            continue
        first = m - n + 1  # keys that the first query sees (none where negative)
        lo = max(first, 0)
        pairs += (m + lo) * (m - lo + 1) // 2 if m >= lo else 0
        keys += m
    return pairs, keys


def work(case):
    if case["op"] == "reserve":
        new, lens, page = _ints(case["new"]), _ints(case["lens"]), case["page"]
        ended = _ended(case)
        base = [0 if e else m for e, m in zip(ended, lens)]
        pages = sum(_ceil(b + n, page) - _ceil(b, page) for b, n in zip(base, new))
        back = sum(_ceil(m, page) for e, m in zip(ended, lens) if e)
        # offsets, lengths in and out, starts, marks; pages read and written; a slot a row
        return {"bytes": 4 * (4 * len(new) + 1) + len(new) + 8 * (pages + back) + 4 * sum(new), "flops": 0}
    if case["op"] == "append":
        return {"bytes": case["rows"] * (case["kv_heads"] * HEAD_DIM * 2 * (2 + _width(case)) + 4) + 4 * case["pad"],
                "flops": 0}
    pairs, keys = _visible(case)
    rows = sum(_ints(case["new"]))
    return {"bytes": 2 * rows * case["heads"] * HEAD_DIM * 2 + keys * (2 * case["kv_heads"] * HEAD_DIM * _width(case)),
            "flops": 4 * HEAD_DIM * case["heads"] * pairs}


def _width(case):
    return 1 if case["dtype"] == "e4m3" else 2


def _ended(case):
    """Every k-th place in the batch is handed on, `ended` of them."""
    b = len(_ints(case["new"]))
    step = max(1, b // max(1, case["ended"]))
    return [i % step == 0 and i // step < case["ended"] for i in range(b)]


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


def prepare(case, seed):
    cpu = torch.Generator().manual_seed(seed)
    gen = torch.Generator(device="cuda").manual_seed(seed)
    s = {"case": case}
    if case["op"] == "reserve":
        new, lens, page = _ints(case["new"]), _ints(case["lens"]), case["page"]
        ended = _ended(case)
        most = max(_ceil(m + n, page) for m, n in zip(lens, new)) + 2
        table, order, at, n_pages = _table(cpu, lens, page, case["spare"], most)
        free = torch.zeros(n_pages, dtype=torch.int32)
        free[:n_pages - at] = order[at:]
        rows = sum(new) + 5  # the rows a host bound allows for
        s.update(table=table, lens=_dev(lens), offsets=_dev(_offsets(new)), free=free.cuda(), count=_dev([n_pages - at]),
                 reset=_dev(ended, torch.uint8), start=_dev([0] * len(new)), lens_out=_dev([0] * len(new)),
                 slots=_dev([0] * rows), count_out=_dev([0]), status=_dev([0]))
        # (the pages themselves are neither read nor written)
        s["k"] = s["v"] = torch.empty((n_pages, 1, page, HEAD_DIM), dtype=torch.bfloat16, device="cuda")
        s["ks"] = s["vs"] = None
        s["first_table"], s["first_free"] = s["table"].clone(), s["free"].clone()
    elif case["op"] == "append":
        rows, pad, page, hkv = case["rows"], case["pad"], case["page"], case["kv_heads"]
        n_pages = _ceil(rows, page) + 9
        s["k"], s["v"], s["ks"], s["vs"] = _pages(case, n_pages, gen)
        order = torch.randperm(n_pages, generator=cpu)
        j = torch.arange(rows) + page // 2  # as if the sequence held half a page before
        slots = torch.cat([order[j // page] * page + j % page, torch.full((pad,), -1)]).to(torch.int32)
        h = case["fused"]
        qkv = torch.randn((rows + pad, h + 2 * hkv, HEAD_DIM), dtype=torch.bfloat16, device="cuda", generator=gen)
        s.update(slots=slots.cuda(), k_new=qkv[:, h:h + hkv], v_new=qkv[:, h + hkv:],
                 table=torch.full((1, 1), -1, dtype=torch.int32, device="cuda"))
    else:
        new, lens, page = _ints(case["new"]), _ints(case["lens"]), case["page"]
        s["table"], _, _, n_pages = _table(cpu, lens, page, 3, max(_ceil(m, page) for m in lens) + 1)
        s["k"], s["v"], s["ks"], s["vs"] = _pages(case, n_pages, gen)
        s["q"] = torch.randn((sum(new), case["heads"], HEAD_DIM), dtype=torch.bfloat16, device="cuda", generator=gen)
        s["o"] = torch.empty_like(s["q"])
        s.update(offsets=_dev(_offsets(new)), lens=_dev(lens), most=max(new), most_keys=max(lens))
    if own:
        import paper_2608_29291_amd as ce
        s["cache"] = ce.KVCache(s["k"], s["v"], s["table"], s["ks"], s["vs"])
        if case["op"] == "attend":
            s["ws"] = ce.alloc_paged_workspace(s["cache"], s["q"].shape[0], case["heads"])
    return s


# ----------------------------------------------------------------- one pass

def run(s):
    op = s["case"]["op"]
    if op == "reserve":
        return _reserve(s)
    return _append(s) if op == "append" else _attend(s)


def _reserve(s):
    if own:
        import paper_2608_29291_amd as ce
        # lengths and the count go to buffers of their own and the same pages are
        # pushed and popped every time, so a pass can be repeated, once a table
        # with handed-on places is put back
        if s["case"]["ended"]:
            s["table"].copy_(s["first_table"])
        ce.ce_kv_reserve(s["cache"], s["lens"], s["offsets"], s["free"], s["count"], s["start"], s["slots"],
                         lens_out=s["lens_out"], free_count_out=s["count_out"], reset=s["reset"], status=s["status"])
        return {"table": s["table"], "free": s["free"], "count": s["count_out"], "lens": s["lens_out"],
                "start": s["start"], "slots": s["slots"], "status": s["status"]}
    page, table, free = s["case"]["page"], s["first_table"], s["first_free"]
    n_pages, width = free.numel(), table.shape[1]
    lens, off, ended = s["lens"].long(), s["offsets"].long(), s["reset"] != 0
    col = torch.arange(width, device=table.device)
    # pages of the ended sequences go back on the stack
    back = torch.where(ended, (lens + page - 1) // page, 0)
    first = s["count"].long() + torch.cumsum(back, 0) - back
    at = torch.where(col < back[:, None], first[:, None] + col, n_pages)
    free = torch.cat([free, free.new_zeros(1)]).scatter(0, at.flatten(), table.flatten())
    count = s["count"].long() + back.sum()
    # and pages for the new rows come from its top
    base, n = torch.where(ended, 0, lens), off[1:] - off[:-1]
    held, need = (base + page - 1) // page, (base + n + page - 1) // page
    need = need - held
    long = held + need > width
    need = torch.where(long, 0, need)
    upto = torch.cumsum(need, 0)
    good = ~long & ((need == 0) | (upto <= count))
    need = torch.where(good, need, 0)
    j = col - held[:, None]
    mine = (j >= 0) & (j < need[:, None])
    taken = free[(count - 1 - (upto - need)[:, None] - j).clamp(0, n_pages)]
    table = torch.where(mine, taken, table)
    rows = torch.arange(s["slots"].numel(), device=table.device)
    b = torch.searchsorted(off[1:].contiguous(), rows, right=True).clamp(max=n.numel() - 1)
    pos = base[b] + rows - off[b]
    slot = table[b, (pos // page).clamp(max=width - 1)].long() * page + pos % page
    slot = torch.where(good[b] & (rows < off[-1]), slot, -1)
    short = (~good & ~long).any().int() * 4 + long.any().int() * 8
    i32 = torch.int32
    return {"table": table, "free": free[:n_pages], "count": (count - need.sum()).to(i32),
            "lens": (base + torch.where(good, n, 0)).to(i32), "start": torch.where(good, base, -1).to(i32),
            "slots": slot.to(i32), "status": short.to(i32)[None]}


def _append(s):
    if own:
        import paper_2608_29291_amd as ce
        ce.ce_kv_append(s["cache"], s["k_new"], s["v_new"], s["slots"])
        return {"k": s["k"], "v": s["v"]}
    page = s["case"]["page"]
    slots = s["slots"].long()
    # rows without a slot write the first row once more
    src = torch.where(slots < 0, 0, torch.arange(slots.numel(), device=slots.device))
    at = slots[src]
    for pool, new, scale in ((s["k"], s["k_new"], s["ks"]), (s["v"], s["v_new"], s["vs"])):
        new = new[src]
        if scale is not None:
            pool, new = pool.view(torch.uint8), _quantize(new, scale[:, None]).view(torch.uint8)
        pool[at // page, :, at % page] = new
    return {"k": s["k"], "v": s["v"]}


def _attend(s):
    c = s["case"]
    if own:
        import paper_2608_29291_amd as ce
        ce.ce_paged_attention(s["cache"], s["q"], s["o"], s["offsets"], s["lens"], c["causal"], SCALE, ws=s["ws"])
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
    end = (lens - n)[:, None] + i + 1 if c["causal"] else lens[:, None].expand(b, s["most"])
    seen = j < torch.minimum(end, lens[:, None])[:, :, None]  # [B, queries, keys]
    score.masked_fill_(~seen[:, None, None], -math.inf)
    top = score.amax(-1, keepdim=True)
    score.sub_(torch.where(seen.any(-1)[:, None, None, :, None], top, 0.0)).exp_()
    total = score.sum(-1, keepdim=True)
    out = torch.matmul(score.view(b, hkv, -1, width * page), rows(s["v"], s["vs"])).view(b, hkv, g, s["most"], HEAD_DIM)
    out = torch.where(seen.any(-1)[:, None, None, :, None], out / total, 0.0)
    out = out.permute(0, 3, 1, 2, 4).reshape(b * s["most"], h, HEAD_DIM).to(s["q"].dtype)
    # row r of the batch is row r - off[b] of its sequence b
    r = torch.arange(s["q"].shape[0], device=off.device)
    seq = torch.searchsorted(off[1:].contiguous(), r, right=True)
    return out[seq * s["most"] + r - off[seq]]


# ------------------------------------------------------- the definition, 64 bits

def exact(case, seed):
    if case["op"] == "reserve":
        return None  # whole numbers
    s = prepare(case, seed)
    if case["op"] == "append":  # what is stored, before it is rounded
        slots = s["slots"].long()[:case["rows"]]
        out = {}
        for name, new, scale in (("k", s["k_new"], s["ks"]), ("v", s["v_new"], s["vs"])):
            x, pool = new[:case["rows"]].double(), s[name].double()
            if scale is not None:
                x = (x / scale.double()[:, None]).clamp(-E4M3_MAX, E4M3_MAX)
            pool[slots // case["page"], :, slots % case["page"]] = x
            out[name] = pool
        return out
    new, lens, page = _ints(case["new"]), _ints(case["lens"]), case["page"]
    h, hkv = case["heads"], case["kv_heads"]
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    at = 0
    for b, (n, m) in enumerate(zip(new, lens)):
        ids = s["table"][b, :_ceil(m, page)].long()
        for kh in range(hkv):
            kv = []
            for pool, scale in ((s["k"], s["ks"]), (s["v"], s["vs"])):
                x = (pool if scale is None else pool.view(torch.uint8))[ids, kh]
                x = x.double() if scale is None else x.view(pool.dtype).double() * scale[kh].double()
                kv.append(x.reshape(-1, HEAD_DIM)[:m].contiguous())
            for i0 in range(0, n, 1024):
                n1 = min(n, i0 + 1024)
                for hq in range(kh * (h // hkv), (kh + 1) * (h // hkv)):
                    x = torch.matmul(s["q"][at + i0:at + n1, hq].double(), kv[0].t().contiguous()) / math.sqrt(HEAD_DIM)
                    if case["causal"]:
                        last = torch.arange(i0, n1, device="cuda")[:, None] + (m - n)
                        x[torch.arange(m, device="cuda")[None, :] > last] = -math.inf
                    out[at + i0:at + n1, hq] = torch.matmul(torch.nan_to_num(torch.softmax(x, -1), nan=0.0), kv[1])
        at += n
    return out

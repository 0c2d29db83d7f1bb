"""Pages and slots made on the device, and writes into the pages, against the
oracle's list of free pages and its 8-bit rounding; the three calls in a row as a
serving program makes them; captured steps and other streams."""
import numpy as np
import pytest

import oracle
import paged_util as U
from oracle import paged as op

pytestmark = pytest.mark.gpu


class State:
    """A pool with sequences of given lengths and its tables on the device."""

    def __init__(self, lens, page, n_free, width=None, seed=0):
        import torch
        import paper_2608_29291_amd as ce
        rng = np.random.default_rng(seed)
        held = [-(-n // page) for n in lens]
        self.n_pages, self.page, self.lens = sum(held) + n_free, page, list(lens)
        order = rng.permutation(self.n_pages).astype(np.int32)
        self.table = np.full((len(lens), width or max(held) + 3), -9, np.int32)
        at = 0
        for b, n in enumerate(held):
            self.table[b, :n] = order[at:at + n]
            at += n
        self.free = [int(x) for x in order[at:]]
        up = lambda x: torch.from_numpy(np.ascontiguousarray(x)).cuda()
        self.d_table, self.d_lens = up(self.table), up(np.array(lens, np.int32))
        stack = np.full(self.n_pages, -7, np.int32)
        stack[:len(self.free)] = self.free
        self.d_free, self.d_count = up(stack), up(np.array([len(self.free)], np.int32))
        kv = torch.empty(self.n_pages, 1, page, U.DH, dtype=torch.bfloat16, device="cuda")
        self.cache = ce.KVCache(kv, kv, self.d_table)

    def step(self, new, reset=None, capacity=None, in_place=True):
        """One call, checked against the oracle; the state moves on."""
        import torch
        import paper_2608_29291_amd as ce
        B, total = len(new), sum(new)
        off = torch.from_numpy(np.concatenate([[0], np.cumsum(new)]).astype(np.int32)).cuda()
        cap = total + 3 if capacity is None else capacity
        slots = torch.full((cap,), -77, dtype=torch.int32, device="cuda")
        start = torch.full((B,), -77, dtype=torch.int32, device="cuda")
        status = torch.full((1,), 77, dtype=torch.int32, device="cuda")
        lo = self.d_lens if in_place else torch.full_like(self.d_lens, -77)
        co = self.d_count if in_place else torch.full_like(self.d_count, -77)
        rs = None if reset is None else torch.tensor(reset, dtype=torch.uint8).cuda()
        ce.ce_kv_reserve(self.cache, self.d_lens, off, self.d_free, self.d_count, start, slots,
                         lens_out=None if in_place else lo, free_count_out=None if in_place else co, reset=rs,
                         status=status)
        torch.cuda.synchronize()
        lens, st, sl, table, free, refused = op.reserve(self.lens, new, self.page, self.table, self.free, reset)
        h = lambda x: x.cpu().numpy()
        np.testing.assert_array_equal(h(lo), lens)
        np.testing.assert_array_equal(h(start), st)
        np.testing.assert_array_equal(h(slots), sl + [-1] * (cap - total))
        np.testing.assert_array_equal(h(self.d_table), table)
        assert int(co.item()) == len(free)
        np.testing.assert_array_equal(h(self.d_free)[:len(free)], free)
        want = (ce.CE_DEV_NO_PAGES if "pages" in refused else 0) | (ce.CE_DEV_TOO_LONG if "long" in refused else 0)
        assert int(status.item()) == want
        if not in_place:
            self.d_lens.copy_(lo)
            self.d_count.copy_(co)
        self.lens, self.table, self.free = lens, table, free
        return refused


CASES = {  # lengths, new rows, page, free pages
    "one": ([0], [1], 16, 1),
    "none_new": ([5, 20], [0, 0], 16, 2),
    "page_edges": ([15, 16, 17, 0, 31, 32, 33], [1, 1, 1, 16, 1, 17, 0], 16, 9),
    "prompt": ([0, 7], [5000, 1], 16, 400),
    "big_pages": ([300, 0, 255], [1, 700, 2], 256, 8),
    "many_rows": ([0] * 5, [4000, 1, 2176, 0, 300], 64, 200),
}


@pytest.mark.parametrize("in_place", [True, False])
@pytest.mark.parametrize("name", CASES)
def test_reserve(name, in_place):
    lens, new, page, free = CASES[name]
    s = State(lens, page, free)
    s.step(new, capacity=None, in_place=in_place)


@pytest.mark.parametrize("B", [1, 64, 1023, 1024, 1025, 2049, 5000])
def test_reserve_many_sequences(B):
    rng = np.random.default_rng(B)
    lens = [int(x) for x in rng.integers(0, 60, B)]
    s = State(lens, 16, B, width=8, seed=B)
    for i in range(3):
        new = [int(x) for x in rng.choice([0, 1, 1, 1, 5, 17], B)]
        s.step(new, reset=[int(x) for x in rng.random(B) < (0.3 if i else 0.0)])


@pytest.mark.parametrize("B", [7, 1500])
def test_reserve_runs_out_of_pages(B):
    """Sequences behind the first that finds too few pages get none, others still grow in their last page."""
    s = State([3] * B, 16, B // 2, width=20, seed=1)
    refused = s.step([20] * B)
    assert refused.count("pages") == B - B // 2
    s.step([1] * B)  # a row in the page that is there
    s.step([30] + [0] * (B - 1), reset=[1] + [0] * (B - 2) + [1])  # two give theirs back, one grows


def test_reserve_refuses_what_outgrows_the_table():
    s = State([30, 10, 0], 16, 50, width=3, seed=2)
    assert s.step([19, 5, 60]) == ["long", "", "long"]
    assert s.step([18, 5, 48]) == ["", "", ""]


def test_reserve_only_gives_back():
    import torch
    import paper_2608_29291_amd as ce
    s = State([40, 0, 100, 16], 16, 3, seed=3)
    start = torch.empty(4, dtype=torch.int32, device="cuda")
    reset = torch.tensor([1, 1, 0, 1], dtype=torch.uint8).cuda()
    ce.ce_kv_reserve(s.cache, s.d_lens, None, s.d_free, s.d_count, start, None, reset=reset)
    lens, _, _, _, free, _ = op.reserve(s.lens, [0] * 4, 16, s.table, s.free, [1, 1, 0, 1])
    assert s.d_lens.tolist() == lens == [0, 0, 100, 0]
    assert s.d_free.tolist()[:int(s.d_count.item())] == free
    assert start.tolist() == [0, 0, 100, 0]


def test_reserve_on_bad_data():
    """Lengths, counts, offsets and page numbers out of range: clamped, reported, nothing out of bounds."""
    import torch
    import paper_2608_29291_amd as ce
    i32 = lambda x: torch.tensor(x, dtype=torch.int32).cuda()
    for lens, off, count, bit in (([40, 5], [0, 20, 40], 1 << 30, ce.CE_DEV_BAD_CACHE),
                                  ([1 << 30, -4], [0, 1, 2], 2, ce.CE_DEV_BAD_CACHE),
                                  ([40, 5], [0, 30, 20], 4, ce.CE_DEV_BAD_OFFSETS),
                                  ([40, 5], [-8, 1 << 30, 9], 4, ce.CE_DEV_BAD_OFFSETS),
                                  ([40, 5], [3, 3, 4], 4, ce.CE_DEV_BAD_OFFSETS),
                                  ([40, 5], [0, 20, 100], 9, ce.CE_DEV_OVERFLOW)):
        for rows in (41, 5000):  # slots by the same launch and by their own
            s = State([40, 5], 16, 8)
            slots, start, status = i32([9] * rows), i32([0, 0]), i32([0])
            if bit == ce.CE_DEV_OVERFLOW:
                off = [0, 20, rows + 60]
            ce.ce_kv_reserve(s.cache, i32(lens), i32(off), s.d_free, i32([count]), start, slots,
                             lens_out=i32([0, 0]), free_count_out=i32([0]), status=status)
            assert int(status.item()) & bit, (lens, off, count)
            sl = slots.cpu().numpy()
            assert ((sl >= -1) & (sl < s.n_pages * 16)).all()
    # a free stack of nonsense: the rows get no slot
    s = State([16], 16, 4)
    s.d_free.fill_(1 << 29)
    slots, start, status = i32([9] * 3), i32([0]), i32([0])
    ce.ce_kv_reserve(s.cache, s.d_lens, i32([0, 3]), s.d_free, s.d_count, start, slots, status=status)
    assert slots.tolist() == [-1, -1, -1] and int(status.item()) & ce.CE_DEV_BAD_CACHE


@pytest.mark.parametrize("dtype", ["bf16", "e4m3"])
@pytest.mark.parametrize("rows,hkv,page,fused", [(1, 2, 16, 0), (7, 1, 64, 3), (300, 4, 32, 28), (45, 5, 256, 0)])
def test_append(rows, hkv, page, fused, dtype):
    import torch
    import paper_2608_29291_amd as ce
    rng = np.random.default_rng(rows)
    n_pages = rows // page + 3
    x = U.bf16(rng.standard_normal((rows, fused + 2 * hkv, U.DH)) * 2)
    x[0, fused, :12] = [np.nan, np.inf, -np.inf, 0.0, -0.0, 3e38, -3e38, 1e-38, 448.0, 464.0, 465.0, 1e-3]
    x[rows // 2, -1, 3] = np.nan
    slots = rng.permutation(n_pages * page)[:rows].astype(np.int32)
    if rows > 5:
        slots[[2, 4, 5]] = [-1, n_pages * page, -(1 << 31)]
    ok = (slots >= 0) & (slots < n_pages * page)
    shape = (n_pages, hkv, page, U.DH)
    tdt = torch.bfloat16 if dtype == "bf16" else torch.float8_e4m3fn
    bits = torch.int16 if dtype == "bf16" else torch.uint8
    before = torch.from_numpy(rng.integers(0, 100, shape)).to(bits)
    pk, pv = before.clone().cuda(), (before + 1).cuda()
    scale = lambda: None if dtype == "bf16" else torch.from_numpy(rng.uniform(0.01, 0.03, hkv).astype(np.float32)).cuda()
    ks, vs = scale(), scale()
    cache = ce.KVCache(pk.view(tdt), pv.view(tdt), torch.full((1, 1), -1, dtype=torch.int32, device="cuda"), ks, vs)
    xd = torch.from_numpy(x).to(torch.bfloat16).cuda()
    ce.ce_kv_append(cache, xd[:, fused:fused + hkv], xd[:, fused + hkv:], torch.from_numpy(slots).cuda())
    torch.cuda.synchronize()
    for pool, first, part, s in ((pk, before, x[:, fused:fused + hkv], ks), (pv, before + 1, x[:, fused + hkv:], vs)):
        want = first.numpy().copy()
        if dtype == "bf16":
            new = torch.from_numpy(np.ascontiguousarray(part)).to(torch.bfloat16).view(torch.int16).numpy()
        else:
            new = U.quantize(part, s.cpu().numpy())
        for r in np.nonzero(ok)[0]:
            want[slots[r] // page, :, slots[r] % page] = new[r]
        got = pool.cpu().numpy()
        if dtype == "e4m3":  # every NaN is one
            got, want = (np.where((y & 0x7f) == 0x7f, 0x7f, y) for y in (got, want))
        np.testing.assert_array_equal(got, want)


def test_append_every_bf16_value_rounds_as_the_oracle():
    import torch
    import paper_2608_29291_amd as ce
    x = np.arange(65536, dtype=np.uint16).view(np.int16).reshape(256, 2, U.DH)
    xd = torch.from_numpy(x.copy()).view(torch.bfloat16).cuda()
    scale = torch.tensor([1.0, 0.37], device="cuda")
    k = torch.zeros(16, 2, 16, U.DH, dtype=torch.uint8, device="cuda")
    cache = ce.KVCache(k.view(torch.float8_e4m3fn), torch.zeros_like(k).view(torch.float8_e4m3fn),
                       torch.zeros(1, 1, dtype=torch.int32, device="cuda"), scale, scale)
    ce.ce_kv_append(cache, xd, xd, torch.arange(256, dtype=torch.int32, device="cuda"))
    got = k.permute(0, 2, 1, 3).reshape(256, 2, U.DH).cpu().numpy()
    with np.errstate(invalid="ignore"):
        want = U.quantize(xd.float().cpu().numpy(), scale.cpu().numpy())
    nan = (want & 0x7f) == 0x7f
    assert np.array_equal((got & 0x7f) == 0x7f, nan)
    np.testing.assert_array_equal(got[~nan], want[~nan])


class Server:
    """The three calls of a layer as a serving program makes them, beside dense keys and values."""

    def __init__(self, B, page, n_pages, dtype, H=12, Hkv=2, seed=0):
        import torch
        import paper_2608_29291_amd as ce
        self.B, self.page, self.H, self.Hkv, self.dtype = B, page, H, Hkv, dtype
        self.rng = np.random.default_rng(seed)
        dev = dict(device="cuda")
        tdt = torch.bfloat16 if dtype == "bf16" else torch.uint8
        fill = float("nan") if dtype == "bf16" else 0x7f
        k = torch.full((n_pages, Hkv, page, U.DH), fill, dtype=tdt, **dev)
        v = torch.full((n_pages, Hkv, page, U.DH), fill, dtype=tdt, **dev)
        self.ks = self.vs = None
        sc = []
        if dtype == "e4m3":
            k, v = k.view(torch.float8_e4m3fn), v.view(torch.float8_e4m3fn)
            self.ks, self.vs = (self.rng.uniform(0.01, 0.02, Hkv).astype(np.float32) for _ in range(2))
            sc = [torch.from_numpy(x).cuda() for x in (self.ks, self.vs)]
        self.table = torch.full((B, 64), -1, dtype=torch.int32, **dev)
        self.cache = ce.KVCache(k, v, self.table, *sc)
        self.lens = torch.zeros(B, dtype=torch.int32, **dev)
        self.free = torch.from_numpy(self.rng.permutation(n_pages).astype(np.int32)).cuda()
        self.count = torch.full((1,), n_pages, dtype=torch.int32, **dev)
        self.start = torch.zeros(B, dtype=torch.int32, **dev)
        self.dense = [(np.zeros((0, Hkv, U.DH)), np.zeros((0, Hkv, U.DH))) for _ in range(B)]

    def rows(self, n):
        return U.bf16(self.rng.standard_normal((n, self.H + 2 * self.Hkv, U.DH)))

    def enqueue(self, qkv, off, slots, o, reset, ws):
        import paper_2608_29291_amd as ce
        H, Hkv = self.H, self.Hkv
        ce.ce_kv_reserve(self.cache, self.lens, off, self.free, self.count, self.start, slots, reset=reset)
        ce.ce_kv_append(self.cache, qkv[:, H:H + Hkv], qkv[:, H + Hkv:], slots)
        ce.ce_paged_attention(self.cache, qkv[:, :H], o, off, self.lens, True, U.DH ** -0.5, ws=ws)

    def remember(self, x, new, reset):
        """The dense answer for rows x, after the same step."""
        at, out, top = 0, [], []
        for b, n in enumerate(new):
            k, v = ([np.zeros((0, self.Hkv, U.DH))] * 2) if reset[b] else self.dense[b]
            part = x[at:at + n]
            kn, vn = part[:, self.H:self.H + self.Hkv], part[:, self.H + self.Hkv:]
            if self.dtype == "e4m3":
                kn, vn = (op.e4m3_value(U.quantize(y, s)) * s.astype(np.float64)[:, None]
                          for y, s in ((kn, self.ks), (vn, self.vs)))
            k, v = np.concatenate([k, kn]), np.concatenate([v, vn])
            self.dense[b] = (k, v)
            out.append(op.attend(part[:, :self.H], k, v, True, U.DH ** -0.5))
            m = np.abs(v).max((0, 2)) if len(v) else np.zeros(self.Hkv)
            top.append(np.repeat(np.repeat(m, self.H // self.Hkv)[None], n, 0))
            at += n
        return np.concatenate(out), np.concatenate(top)


@pytest.mark.parametrize("dtype,page", [("bf16", 16), ("e4m3", 32)])
def test_serving_steps(dtype, page):
    """Prompts, decodes, a chunk and a place handed on, each step's rows against dense attention."""
    import torch
    s = Server(5, page, 120, dtype)
    steps = [([40, 0, 3, 97, 1], [0] * 5), ([1] * 5, [0] * 5), ([1, 130, 1, 1, 1], [0] * 5),
             ([1, 1, 25, 1, 1], [0, 0, 1, 0, 0]), ([4, 1, 2, 0, 5], [0, 0, 0, 1, 0]), ([1] * 5, [0] * 5)]
    for new, reset in steps:
        x = s.rows(sum(new))
        off = torch.from_numpy(np.concatenate([[0], np.cumsum(new)]).astype(np.int32)).cuda()
        cap = sum(new) + 4
        qkv = torch.full((cap, s.H + 2 * s.Hkv, U.DH), float("nan"), dtype=torch.bfloat16, device="cuda")
        qkv[:len(x)] = torch.from_numpy(x).to(torch.bfloat16).cuda()
        slots = torch.empty(cap, dtype=torch.int32, device="cuda")
        o = torch.empty(cap, s.H, U.DH, dtype=torch.bfloat16, device="cuda")
        s.enqueue(qkv, off, slots, o, torch.tensor(reset, dtype=torch.uint8).cuda(), None)
        torch.cuda.synchronize()
        want, top = s.remember(x, new, reset)
        U.check(o[:len(x)].float().cpu().numpy(), want, top)
        assert s.lens.tolist() == [len(k) for k, _ in s.dense]


def test_retained_rows_of_a_routed_layer_into_the_cache():
    """ce_topk_compact's packed counts, which only the device knows, drive the cache."""
    import torch
    import gpu_util as G
    import paper_2608_29291_amd as ce
    from ce_workloads import small_workload
    wl = small_workload("und", seed=5, dtype="bf16", d=128, F=64, r_c=32, r_e=32, keep=0.4)
    _, l32 = oracle.score(wl.hidden, wl.flags, wl.seq_offsets, wl.t, wl.scorer)
    dw = G.DevWorkload(wl)
    kidx, koff = dw.new_idx()
    ce.ce_topk_compact(dw.batch, G.to_dev(l32.astype(np.float32)), kidx, koff, dw.ws(ce.CE_WS_TOPK))
    s = Server(wl.B, 16, 400, "bf16")
    x = s.rows(dw.cap)
    qkv = torch.from_numpy(x).to(torch.bfloat16).cuda()
    slots = torch.empty(dw.cap, dtype=torch.int32, device="cuda")
    o = torch.empty(dw.cap, s.H, U.DH, dtype=torch.bfloat16, device="cuda")
    s.enqueue(qkv, koff, slots, o, None, None)
    torch.cuda.synchronize()
    offs = oracle.select(l32, wl.flags, wl.seq_offsets, wl.keep)["kept_offsets"]
    new = [int(n) for n in np.diff(offs)]
    want, top = s.remember(x[:sum(new)], new, [0] * wl.B)
    U.check(o[:sum(new)].float().cpu().numpy(), want, top)


def test_captured_decode_steps():
    """A decode step captured once and replayed: the cache grows in place."""
    import torch
    import paper_2608_29291_amd as ce
    s = Server(6, 16, 200, "bf16", seed=3)
    new = [700, 3, 15, 16, 1, 260]
    x = s.rows(sum(new))
    off = torch.from_numpy(np.concatenate([[0], np.cumsum(new)]).astype(np.int32)).cuda()
    o = torch.empty(sum(new), s.H, U.DH, dtype=torch.bfloat16, device="cuda")
    s.enqueue(torch.from_numpy(x).to(torch.bfloat16).cuda(), off, torch.empty(sum(new), dtype=torch.int32, device="cuda"),
              o, None, None)
    s.remember(x, new, [0] * 6)
    off1 = torch.arange(7, dtype=torch.int32, device="cuda")
    qkv = torch.zeros(6, s.H + 2 * s.Hkv, U.DH, dtype=torch.bfloat16, device="cuda")
    slots = torch.empty(6, dtype=torch.int32, device="cuda")
    o1 = torch.empty(6, s.H, U.DH, dtype=torch.bfloat16, device="cuda")
    ws = ce.alloc_paged_workspace(s.cache, 6, s.H)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        s.enqueue(qkv, off1, slots, o1, None, ws)
    for i in range(20):
        x = s.rows(6)
        qkv.copy_(torch.from_numpy(x).to(torch.bfloat16))
        graph.replay()
        torch.cuda.synchronize()
        want, top = s.remember(x, [1] * 6, [0] * 6)
        U.check(o1.float().cpu().numpy(), want, top, f"replay {i}")
        if i == 10:  # an eager step in between
            x = s.rows(6)
            qkv.copy_(torch.from_numpy(x).to(torch.bfloat16))
            s.enqueue(qkv, off1, slots, o1, None, ws)
            torch.cuda.synchronize()
            want, top = s.remember(x, [1] * 6, [0] * 6)
            U.check(o1.float().cpu().numpy(), want, top, "eager step")


def test_other_streams():
    """Two calls on streams of their own, with scratch of their own, and a raw stream handle."""
    import torch
    new, lens = [1, 1], [3000, 2000]
    p = U.Paged(lens, 2, 16, "bf16", seed=21)
    q = U.bf16(np.random.default_rng(1).standard_normal((2, 12, U.DH)))
    first = U.attend(p, q, new, True)
    c = p.cache()
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]

    class Raw:
        cuda_stream = streams[0].cuda_stream

    for st in (*streams, Raw()):
        got = U.attend(p, q, new, True, cache=c, ws=False, stream=st)
        assert np.array_equal(got, first)

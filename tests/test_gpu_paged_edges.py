"""The paged cache where its documentation allows what other tests do not reach: pools
past 4 GiB, several tiles of a sequence in a batch of single tokens, wide head groups, calls
captured and replayed that share a workspace, calls with nothing to do, wrong offsets
of every batch size, scales at the ends of their range."""
import numpy as np
import pytest

import paged_util as U

pytestmark = pytest.mark.gpu


def rows(new, heads, seed=1):
    return U.bf16(np.random.default_rng(seed).standard_normal((sum(new), heads, U.DH)))


def i32(x):
    import torch
    return torch.tensor(x, dtype=torch.int32).cuda()


@pytest.mark.parametrize("dtype", ["bf16", "e4m3"])
@pytest.mark.parametrize("B", [40, 200, 300])
def test_several_tiles_of_a_sequence_among_single_tokens(B, dtype):
    """No more rows than sequences, most of them one sequence's: tiles of 32 rows, their
    causal edges and the chunks that meet."""
    new = [0] * B
    new[B // 3], new[-1], new[0] = 30, 1, 1
    lens = [0] * B
    lens[B // 3], lens[-1], lens[0], lens[1] = 2777, 1200, 1, 77
    p = U.Paged(lens, 4, 16, dtype, seed=B)
    q = rows(new, 28)
    for causal in (True, False):
        U.check(U.attend(p, q, new, causal), *p.answer(q, new, causal, U.DH ** -0.5))


@pytest.mark.parametrize("H,Hkv,new,lens", [(40, 1, [1, 3], [900, 40]), (4096, 1, [1, 2], [90, 300]),
                                            (66, 2, [2, 1], [700, 129]), (45, 45, [1, 2, 1], [20, 600, 1])])
@pytest.mark.parametrize("dtype", ["bf16", "e4m3"])
def test_head_groups(H, Hkv, new, lens, dtype):
    """More heads a key/value head than rows of a tile, and as many of both."""
    p = U.Paged(lens, Hkv, 32, dtype, seed=H)
    q = rows(new, H)
    U.check(U.attend(p, q, new, True), *p.answer(q, new, True, U.DH ** -0.5))


@pytest.mark.parametrize("dtype", ["bf16", "e4m3"])
def test_pools_past_four_gib(dtype):
    """Pages whose offsets need more than 32 bits, written and read."""
    import torch
    import paper_2608_29291_amd as ce
    Hkv, page, new = 2, 16, [1, 40, 1]
    lens = [700, 333, 15]
    p = U.Paged(lens, Hkv, page, dtype, seed=31)
    apart = 8 if dtype == "bf16" else 16  # layers that share the allocation: 64 KB a page
    n = (1 << 32) // 65536 + 1000
    tdt = torch.bfloat16 if dtype == "bf16" else torch.float8_e4m3fn
    k, v = (torch.empty(n, apart, Hkv, page, U.DH, dtype=tdt, device="cuda")[:, apart - 1] for _ in range(2))
    c0 = p.cache()
    table = torch.where(c0.page_table < p.n_pages, c0.page_table + (n - p.n_pages), c0.page_table)
    c = ce.KVCache(k, v, table, c0.k_scale, c0.v_scale)
    slots, kn, vn = [], [], []
    for b, m in enumerate(lens):
        slots += [int(p.table[b, j // page] + n - p.n_pages) * page + j % page for j in range(m)]
        kn.append(p.k[b])
        vn.append(p.v[b])
    up = lambda x: torch.from_numpy(np.concatenate(x)).to(torch.bfloat16).cuda()
    ce.ce_kv_append(c, up(kn), up(vn), i32(slots))
    q = rows(new, 12)
    got = U.attend(p, q, new, True, cache=c)
    U.check(got, *p.answer(q, new, True, U.DH ** -0.5))


@pytest.mark.parametrize("B", [5, 300])
def test_captured_calls_share_a_workspace_in_turn(B):
    """A graph of single tokens and one of many rows, replayed in turn with eager calls
    between them, on one workspace, with lengths that grow."""
    import torch
    import paper_2608_29291_amd as ce
    lens = [0] * B
    lens[0], lens[1], lens[2], lens[-1] = 5000, 1300, 40, 900
    p = U.Paged(lens, 2, 16, "bf16", seed=41)
    c = p.cache()
    H, kinds = 12, []
    for new in ([1] * 3 + [0] * (B - 4) + [1], [1, 150, 40] + [0] * (B - 4) + [3]):
        q = torch.zeros(sum(new), H, U.DH, dtype=torch.bfloat16, device="cuda")
        kinds.append((new, q, torch.zeros_like(q), i32([0] + np.cumsum(new).tolist()), i32(lens)))
    ws = ce.alloc_paged_workspace(c, sum(kinds[1][0]), H)
    ws.fill_(0xff)
    call = lambda x: ce.ce_paged_attention(c, x[1], x[2], x[3], x[4], True, U.DH ** -0.5, ws=ws)
    torch.cuda.synchronize()
    graphs = []
    for x in kinds:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            call(x)
        graphs.append(g)
    for i in range(6):
        x, g = kinds[i % 2], graphs[i % 2]
        q = rows(x[0], H, seed=i)
        x[1].copy_(torch.from_numpy(q).to(torch.bfloat16))
        now = [max(n - 37 * (5 - i), m) if n else 0 for n, m in zip(lens, x[0])]
        x[4].copy_(i32(now))
        p2k, p2v = p.k_used, p.v_used
        p.k_used, p.v_used = [y[:m] for y, m in zip(p2k, now)], [y[:m] for y, m in zip(p2v, now)]
        want, top = p.answer(q, x[0], True, U.DH ** -0.5)
        p.k_used, p.v_used = p2k, p2v
        for run in (g.replay, g.replay, lambda: call(x), g.replay):
            x[2].fill_(7.0)
            run()
            torch.cuda.synchronize()
            U.check(x[2].float().cpu().numpy(), want, top, f"step {i}")


def test_nothing_to_do():
    import torch
    import paper_2608_29291_amd as ce
    p = U.Paged([40, 0], 2, 16, "bf16", seed=51)
    c = p.cache()
    before = c.k.clone().view(torch.int16)
    none = torch.empty(0, 2, U.DH, dtype=torch.bfloat16, device="cuda")
    empty = torch.empty(0, dtype=torch.int32, device="cuda")
    ce.ce_kv_append(c, none, none, empty)
    q = torch.empty(0, 4, U.DH, dtype=torch.bfloat16, device="cuda")
    ce.ce_paged_attention(c, q, torch.empty_like(q), i32([0, 0, 0]), i32([40, 0]), True, 1.0)
    # room for rows, and none there: what stands in the outputs stays
    q = torch.randn(9, 4, U.DH, dtype=torch.bfloat16, device="cuda")
    o = torch.full_like(q, 77.0)
    ce.ce_paged_attention(c, q, o, i32([0, 0, 0]), i32([40, 0]), True, 1.0)
    lens, count = i32([40, 0]), i32([2])
    free, start, slots, status = i32([0] * p.n_pages), i32([9, 9]), i32([9] * 5), i32([9])
    ce.ce_kv_reserve(c, lens, i32([0, 0, 0]), free, count, start, slots, status=status)
    ce.ce_kv_append(c, torch.randn(5, 2, U.DH, device="cuda").bfloat16(), torch.randn(5, 2, U.DH, device="cuda").bfloat16(),
                    slots)
    torch.cuda.synchronize()
    assert (o == 77.0).all() and torch.equal(c.k.view(torch.int16), before)
    assert lens.tolist() == [40, 0] and count.item() == 2 and start.tolist() == [40, 0]
    assert slots.tolist() == [-1] * 5 and status.item() == 0


@pytest.mark.parametrize("B", [3, 70, 300])
@pytest.mark.parametrize("dtype", ["bf16", "e4m3"])
def test_wrong_offsets_stay_in_bounds(B, dtype):
    """Offsets out of order, negative or past the rows, in batches planned by one wave, by
    four sequences a lane and by their own launch, of single tokens and of many
    rows; the same workspace then serves a right call."""
    import torch
    import paper_2608_29291_amd as ce
    rng = np.random.default_rng(B)
    lens = [int(x) for x in rng.integers(0, 60, B)]
    lens[0], lens[B // 2] = 1500, 800
    p = U.Paged(lens, 2, 16, dtype, seed=B)
    c = p.cache()
    for n in (B, 6 * B):  # (8 heads: four a key/value head)
        q = torch.randn(n, 8, U.DH, dtype=torch.bfloat16, device="cuda")
        o = torch.empty(n + 1, 8, U.DH, dtype=torch.bfloat16, device="cuda").fill_(77.0)
        ws = ce.alloc_paged_workspace(c, n, 8)
        size = ws.numel()
        guard = torch.full((size + 4096,), 0xa5, dtype=torch.uint8, device="cuda")
        ws = guard[:size]
        for off in (rng.integers(-5, n + 9, B + 1), np.where(np.arange(B + 1) % 2, n, 0), np.arange(B, -1, -1) * n // B,
                    rng.integers(-(1 << 31), 1 << 31, B + 1)):
            for m in (lens, rng.integers(-(1 << 31), 1 << 31, B)):
                ce.ce_paged_attention(c, q, o[:n], i32(np.asarray(off).tolist()), i32(np.asarray(m).tolist()), True,
                                      U.DH ** -0.5, ws=ws)
                torch.cuda.synchronize()
                assert (o[n] == 77.0).all() and (guard[size:] == 0xa5).all()
        new = [1] * B if n == B else [6] * B
        want, top = p.answer(q.float().cpu().numpy(), new, True, U.DH ** -0.5)
        ce.ce_paged_attention(c, q, o[:n], i32([0] + np.cumsum(new).tolist()), i32(lens), True, U.DH ** -0.5, ws=ws)
        U.check(o[:n].float().cpu().numpy(), want, top)


@pytest.mark.parametrize("total", [100, 6000])
def test_rows_before_the_first_offset_get_no_slot(total):
    import torch
    import paper_2608_29291_amd as ce
    k = torch.empty(500, 1, 16, U.DH, dtype=torch.bfloat16, device="cuda")
    c = ce.KVCache(k, k, torch.zeros(2, 400, dtype=torch.int32, device="cuda"))
    slots, status = torch.full((total,), 9, dtype=torch.int32, device="cuda"), i32([0])
    ce.ce_kv_reserve(c, i32([0, 0]), i32([7, 30, 50]), torch.arange(500, dtype=torch.int32, device="cuda"), i32([500]),
                     i32([0, 0]), slots, lens_out=i32([0, 0]), free_count_out=i32([0]), status=status)
    s = slots.cpu().numpy()
    assert (s[:7] == -1).all() and (s[7:50] >= 0).all() and (s[50:] == -1).all()
    assert status.item() == ce.CE_DEV_BAD_OFFSETS


@pytest.mark.parametrize("scale", [1e-36, 9e-31, 9e-25, 1.1e-24, 2.0 ** -20, 2.0 ** 20, 9e23, 1.1e24, 1e36])
def test_scales_far_from_one(scale):
    """Values of the scale's size: quotients over the whole range of the format."""
    import torch
    import paper_2608_29291_amd as ce
    rng = np.random.default_rng(3)
    s = np.array([scale, scale * 1.37], np.float32)
    x = U.bf16(rng.standard_normal((64, 2, U.DH)) * np.exp2(rng.uniform(-11, 9.5, (64, 2, U.DH))) * s[0])
    x[0, :, :4] = [0.0, -0.0, np.inf, np.nan]
    k = torch.zeros(4, 2, 16, U.DH, dtype=torch.uint8, device="cuda")
    v = torch.zeros_like(k)
    sd = torch.from_numpy(s).cuda()
    c = ce.KVCache(k.view(torch.float8_e4m3fn), v.view(torch.float8_e4m3fn), i32([[0]]), sd, sd)
    xd = torch.from_numpy(x).to(torch.bfloat16).cuda()
    ce.ce_kv_append(c, xd, xd, torch.arange(64, dtype=torch.int32, device="cuda"))
    want = U.quantize(x, s)
    for pool in (k, v):
        got = pool.permute(0, 2, 1, 3).reshape(64, 2, U.DH).cpu().numpy()
        nan = (want & 0x7f) == 0x7f
        assert np.array_equal((got & 0x7f) == 0x7f, nan)
        np.testing.assert_array_equal(got[~nan], want[~nan])


@pytest.mark.parametrize("dtype", ["bf16", "e4m3"])
def test_rows_with_one_slot(dtype):
    """Each 16 bytes of the page come from one of the rows."""
    import torch
    import paper_2608_29291_amd as ce
    n, Hkv = 500, 4
    x = U.bf16(np.random.default_rng(5).integers(-8, 9, (n, Hkv, U.DH)))
    bits = torch.int16 if dtype == "bf16" else torch.uint8
    k = torch.zeros(2, Hkv, 16, U.DH, dtype=bits, device="cuda")
    v = torch.zeros_like(k)
    tdt = torch.bfloat16 if dtype == "bf16" else torch.float8_e4m3fn
    c = ce.KVCache(k.view(tdt), v.view(tdt), i32([[0]]))
    xd = torch.from_numpy(x).to(torch.bfloat16).cuda()
    ce.ce_kv_append(c, xd, xd, i32([21] * n))
    per = 8 if dtype == "bf16" else 16
    cand = x.reshape(n, Hkv, U.DH // per, per)
    for pool in (k, v):
        got = pool.view(tdt)[1, :, 5].float().cpu().numpy().reshape(1, Hkv, U.DH // per, per)
        assert (cand == got).all(-1).any(0).all()
        pool[1, :, 5] = 0
        assert not pool.any()  # and nothing else


@pytest.mark.parametrize("dtype", ["bf16", "e4m3"])
def test_pages_without_scales(dtype):
    p = U.Paged([700, 50], 2, 16, dtype, seed=61, scales=False)
    for new in ([1, 1], [50, 7]):
        q = rows(new, 12)
        U.check(U.attend(p, q, new, True), *p.answer(q, new, True, U.DH ** -0.5))


def test_refusals_of_the_binding():
    """Workspaces that are too small or misaligned, vectors that are too short, rows that differ."""
    import torch
    import paper_2608_29291_amd as ce
    p = U.Paged([700, 50], 2, 16, "bf16", seed=71)
    c = p.cache()
    q = torch.zeros(90, 12, U.DH, dtype=torch.bfloat16, device="cuda")
    o, off, lens = torch.zeros_like(q), i32([0, 1, 90]), i32([700, 50])
    ws = ce.alloc_paged_workspace(c, 90, 12)
    go = lambda **kw: ce.ce_paged_attention(c, *(kw.get(n, x) for n, x in (("q", q), ("o", o), ("off", off), ("lens", lens))),
                                            True, kw.get("scale", 0.1), ws=kw.get("ws", ws))
    go()
    for kw in ({"ws": ws[:-256]}, {"ws": ws[16:]}, {"off": off[:2]}, {"lens": lens[:1]}, {"o": o[:89]},
               {"o": torch.zeros(90, 13, U.DH, dtype=torch.bfloat16, device="cuda")[:, :12]}, {"q": q.float()},
               {"q": q[:, :11]}, {"q": q.cpu()}, {"off": off.long()}, {"scale": 0.0}):
        with pytest.raises((ValueError, ce.CERouterError)):
            go(**kw)
    k = torch.zeros(9, 2, U.DH, dtype=torch.bfloat16, device="cuda")
    for args in ((k, k[:8], i32([0] * 9)), (k, k, i32([0] * 8)), (k[:, :1], k, i32([0] * 9)), (k, k.float(), i32([0] * 9))):
        with pytest.raises((ValueError, ce.CERouterError)):
            ce.ce_kv_append(c, *args)
    free, count, start, slots = i32([0] * p.n_pages), i32([0]), i32([0, 0]), i32([0] * 9)
    for args in ((lens[:1], off, free, count, start, slots), (lens, off[:2], free, count, start, slots),
                 (lens, off, free[:-1], count, start, slots), (lens, None, free, count, start, slots),
                 (lens, off, free, count, start[:1], slots), (lens, off, free, count, start, slots.long())):
        with pytest.raises((ValueError, ce.CERouterError)):
            ce.ce_kv_reserve(c, *args)
    torch.cuda.synchronize()


@pytest.mark.parametrize("dtype", ["bf16", "e4m3"])
def test_rows_past_four_gib(dtype):
    """Queries and outputs whose offsets need more than 32 bits, behind rows that see no token."""
    import torch
    import paper_2608_29291_amd as ce
    H, Hkv, first = 64, 8, 270000
    new, lens = [0, 40, 1], [0, 300, 777]
    p = U.Paged(lens, Hkv, 16, dtype, seed=81)
    c = p.cache()
    n = first + sum(new)
    q = torch.full((n, H, U.DH), 0.5, dtype=torch.bfloat16, device="cuda")
    o = torch.full_like(q, 77.0)
    x = rows(new, H)
    q[first:] = torch.from_numpy(x).to(torch.bfloat16).cuda()
    ce.ce_paged_attention(c, q, o, i32([0, first, first + 40, n]), i32(lens), True, U.DH ** -0.5)
    U.check(o[first:].float().cpu().numpy(), *p.answer(x, new, True, U.DH ** -0.5))
    assert not o[:first:1000].any() and not o[first - 1].any()


def test_most_sequences():
    """The largest batch, one token each, all over the same few pages."""
    import torch
    import paper_2608_29291_amd as ce
    B, H, Hkv = 65535, 6, 2
    p = U.Paged([160], Hkv, 16, "bf16", seed=91)
    lens = np.random.default_rng(2).integers(0, 161, B)
    p.table = np.repeat(p.table, B, 0)
    q = rows([B], H)
    qd = torch.from_numpy(q).to(torch.bfloat16).cuda()
    o = torch.full_like(qd, 77.0)
    ce.ce_paged_attention(p.cache(), qd, o, torch.arange(B + 1, dtype=torch.int32, device="cuda"), i32(lens.tolist()), True,
                          U.DH ** -0.5)
    got = o.float().cpu().numpy()
    assert not (got == 77.0).all((1, 2)).any()
    k, v = p.k_used[0], p.v_used[0]
    for b in (0, 1, 255, 256, 511, 4095, 4096, 40000, B - 1):
        p.k_used, p.v_used = [k[:lens[b]]], [v[:lens[b]]]
        U.check(got[b:b + 1], *p.answer(q[b:b + 1], [1], True, U.DH ** -0.5))


def test_every_sequence_of_the_largest_batch_gets_a_page():
    import torch
    import paper_2608_29291_amd as ce
    B = 65535
    k = torch.empty(B + 5, 1, 16, U.DH, dtype=torch.bfloat16, device="cuda")
    c = ce.KVCache(k, k, torch.full((B, 2), -1, dtype=torch.int32, device="cuda"))
    lens, count, status = torch.zeros(B, dtype=torch.int32, device="cuda"), i32([B + 5]), i32([9])
    start, slots = torch.full_like(lens, 9), torch.full_like(lens, 9)
    free = torch.arange(B + 5, dtype=torch.int32, device="cuda")
    ce.ce_kv_reserve(c, lens, torch.arange(B + 1, dtype=torch.int32, device="cuda"), free, count, start, slots, status=status)
    page = torch.arange(B + 4, 4, -1, dtype=torch.int32, device="cuda")  # from the top of the stack
    assert torch.equal(c.page_table[:, 0], page) and (c.page_table[:, 1] == -1).all()
    assert torch.equal(slots, page * 16) and not start.any() and (lens == 1).all()
    assert count.item() == 5 and status.item() == 0

"""Steps of drafted decoding as a program makes them: reserve, masks, rotary, append, attention,
verification, keep and trim, several steps long, over two layers that share a page table; and
the same steps captured in a graph."""
import numpy as np
import pytest
import torch

import draft_util as du
import paged_util as pu
from oracle import draft as od

pytestmark = pytest.mark.gpu
ce = pytest.importorskip("paper_2608_29291_amd")

LAYERS, HKV, H, PAGE, VOCAB, FREQ = 2, 2, 6, 16, 3000, 32


class Program:
    """What a serving program keeps, and one step of it."""

    def __init__(self, B, rows, n_pages, width, words, seed):
        self.rng = np.random.default_rng(seed)
        self.B, self.rows, self.words = B, rows, words
        i32 = lambda *s, v=0: torch.full(s, v, dtype=torch.int32, device="cuda")
        pool = lambda: torch.zeros((n_pages, HKV, PAGE, du.DH), dtype=torch.bfloat16, device="cuda")
        self.table = i32(B, width, v=-1)
        self.caches = [ce.KVCache(pool(), pool(), self.table) for _ in range(LAYERS)]
        self.lens, self.free = i32(B), torch.arange(n_pages, dtype=torch.int32, device="cuda")
        self.count, self.start, self.slots = i32(1, v=n_pages), i32(B), i32(rows)
        self.off, self.parents, self.tokens = i32(B + 1), i32(rows), i32(rows)
        self.mask, self.positions, self.base = i32(rows, words), i32(rows), i32(B)
        self.kept, self.n_kept, self.next = i32(rows), i32(B), i32(B)
        self.qkv = [torch.zeros((rows, H + 2 * HKV, du.DH), dtype=torch.bfloat16, device="cuda") for _ in range(LAYERS)]
        self.o = [torch.zeros((rows, H, du.DH), dtype=torch.bfloat16, device="cuda") for _ in range(LAYERS)]
        self.logits = torch.zeros((rows, VOCAB), dtype=torch.bfloat16, device="cuda")
        self.u = torch.zeros(rows, device="cuda")
        self.drafts = ce.Drafts(self.off, self.parents, self.tokens)
        self.rotary = ce.Rotary(ce.rotary_freqs(2 * FREQ))
        self.ws = ce.alloc_paged_workspace(self.caches[0], rows, H)
        self.vws = ce.alloc_verify_workspace(self.drafts, VOCAB, False)

    def load(self, trees):
        """A step's inputs, of the same sizes every time."""
        new = [len(t) for t in trees]
        n = sum(new)
        host = {"off": du.offsets(new), "parents": np.array([p for t in trees for p in t], np.int32),
                "tokens": self.rng.integers(0, VOCAB, n).astype(np.int32)}
        x = self.rng.standard_normal((n, VOCAB))
        at = 0
        for t in trees:
            for i, p in enumerate(t):
                if p >= 0:
                    x[at + p, host["tokens"][at + i]] = 9 + self.rng.standard_normal()
            at += len(t)
        host["u"] = self.rng.random(n).astype(np.float32)
        host["logits"] = pu.bf16(x)
        host["qkv"] = [pu.bf16(self.rng.standard_normal((n, H + 2 * HKV, du.DH))) for _ in range(LAYERS)]
        self.off.copy_(torch.from_numpy(host["off"]))
        for name in ("parents", "tokens", "u"):
            getattr(self, name)[:n].copy_(torch.from_numpy(host[name]))
        self.logits[:n].copy_(torch.from_numpy(host["logits"]))
        for d, x in zip(self.qkv, host["qkv"]):
            d[:n].copy_(torch.from_numpy(x))
        return host

    def step(self):
        ce.ce_kv_reserve(self.caches[0], self.lens, self.off, self.free, self.count, self.start, self.slots)
        ce.ce_draft_masks(self.drafts, self.mask, positions=self.positions, base=self.base)
        for c, qkv, o in zip(self.caches, self.qkv, self.o):
            turned = qkv[:, :H + HKV]
            ce.ce_rotary(self.rotary, turned, turned, self.positions)
            ce.ce_kv_append(c, qkv[:, H:H + HKV], qkv[:, H + HKV:], self.slots)
            ce.ce_paged_tree_attention(c, qkv[:, :H], o, self.off, self.lens, self.mask, du.DH ** -0.5, ws=self.ws)
        ce.ce_verify_drafts(self.drafts, self.logits, self.u, self.kept, self.n_kept, self.next, ws=self.vws)
        for c in self.caches:
            ce.ce_kv_keep(c, self.off, self.start, self.kept, self.n_kept)
        ce.ce_kv_trim(self.caches[0], self.lens, self.start, self.n_kept, self.free, self.count)
        self.base.add_(self.n_kept)


def check_step(p, host, trees, held, base):
    """The step's outputs, from dense lists of keys and values (held[layer][sequence]), which grow."""
    at = 0
    for b, t in enumerate(trees):
        n = len(t)
        seen, depth = od.masks(t)
        pos = (depth + base[b])[None].astype(np.int64)
        s = slice(at, at + n)
        walk, token = od.verify(t, host["tokens"][s], host["logits"][s].astype(np.float64), 1.0, host["u"][s])
        if n == 0:
            assert int(p.n_kept[b]) == 0 and int(p.next[b]) == -1
            continue
        assert int(p.n_kept[b]) == len(walk) and int(p.next[b]) == token, b
        assert p.kept[s].tolist() == walk + [-1] * (n - len(walk)), b
        for layer in range(LAYERS):
            qkv = host["qkv"][layer][s]
            # (the library's rounding of the turned values counts as input of what follows; it is off by
            # 2^-8 of half a step and 2^-21 of the angle)
            turned = p.turned[layer][s]
            want = od.rotary(qkv[:, :H + HKV], pos, ce.rotary_freqs(2 * FREQ), [0] * FREQ, False)
            assert np.abs(turned - want).max() <= (2.0 ** -9 + 2.0 ** -20) * 2 * 1.5 * np.abs(qkv).max()
            k, v = held[layer][b]
            k = np.concatenate([k, turned[:, H:]])
            v = np.concatenate([v, qkv[:, H + HKV:]])
            o = p.o[layer][s].float().cpu().numpy()
            full = np.concatenate([np.ones((n, len(k) - n), bool), seen], 1)
            want = od.attend(turned[:, :H], k, v, full, du.DH ** -0.5)
            pu.check(o, want, np.full(o.shape[:2], np.abs(v).max()))
            keep = list(range(len(k) - n)) + [len(k) - n + r for r in walk]
            held[layer][b] = k[keep], v[keep]
        base[b] += len(walk)
        at += n
    lens = [len(held[0][b][0]) for b in range(p.B)]
    assert p.lens.tolist() == lens
    # the cache holds the accepted rows and nothing is lost of the pool
    table, free = p.table.cpu().numpy(), p.free[:int(p.count)].tolist()
    used = [int(table[b, j]) for b, m in enumerate(lens) for j in range(-(-m // PAGE))]
    assert sorted(used + free) == list(range(p.free.numel()))
    for layer, c in enumerate(p.caches):
        ck, cv = c.k.float().cpu().numpy(), c.v.float().cpu().numpy()
        for b, m in enumerate(lens):
            for pool, want in zip((ck, cv), held[layer][b]):
                got = [pool[table[b, j // PAGE], :, j % PAGE] for j in range(m)]
                assert m == 0 or np.array_equal(np.array(got), want), (layer, b)


def empty(B):
    z = lambda: np.zeros((0, HKV, du.DH), np.float32)
    return [[(z(), z()) for _ in range(B)] for _ in range(LAYERS)]


def turned_rows(p, n):
    p.turned = [x[:n, :H + HKV].float().cpu().numpy() for x in p.qkv]


def test_steps():
    p = Program(4, 120, 40, 12, 2, seed=0)
    held, base = empty(4), [0] * 4
    for i, new in enumerate([(40, 1, 17, 0), (9, 26, 33, 5), (1, 1, 1, 1), (20, 50, 0, 34), (26, 26, 26, 26)]):
        trees = [list(range(-1, n - 1)) if i == 0 else du.tree(p.rng, n, 0.5) if n else [] for n in new]
        host = p.load(trees)
        p.step()
        torch.cuda.synchronize()
        turned_rows(p, sum(new))
        check_step(p, host, trees, held, base)


def test_captured_steps():
    """One graph, replayed with new trees each time, eager work of the same program between."""
    shapes = [(9, 26, 33), (12, 5, 40), (33, 26, 9), (20, 20, 20), (1, 1, 1)]
    p = Program(3, 70, 60, 20, 2, seed=3)
    p.load([du.tree(p.rng, n) for n in shapes[0]])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    saved = [t.clone() for t in (p.lens, p.count, p.free, p.table, p.base)]
    with torch.cuda.stream(side):
        p.step()  # (modules are loaded before the capture)
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    for t, s in zip((p.lens, p.count, p.free, p.table, p.base), saved):
        t.copy_(s)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        p.step()
    held, base = empty(3), [0] * 3
    for i, new in enumerate(shapes * 2):
        trees = [du.tree(p.rng, n, 0.5) for n in new]
        host = p.load(trees)
        if i % 3 == 1:
            p.step()
        else:
            graph.replay()
        torch.cuda.synchronize()
        turned_rows(p, sum(new))
        check_step(p, host, trees, held, base)


def test_two_captured_graphs_with_workspaces_of_their_own():
    ps = [Program(2, 70, 40, 20, 2, seed=s) for s in (5, 6)]
    graphs, hosts, trees = [], [], []
    for p in ps:
        trees.append([du.tree(p.rng, n) for n in (33, 30)])
        hosts.append(p.load(trees[-1]))
        saved = [t.clone() for t in (p.lens, p.count, p.free, p.table, p.base)]
        p.step()
        torch.cuda.synchronize()
        for t, s in zip((p.lens, p.count, p.free, p.table, p.base), saved):
            t.copy_(s)
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            p.step()
        graphs.append(g)
    held, base = [empty(2) for _ in ps], [[0, 0] for _ in ps]
    streams = [torch.cuda.Stream() for _ in ps]
    for i in range(3):
        for k, p in enumerate(ps):
            trees[k] = [du.tree(p.rng, n) for n in (33, 30)]
            hosts[k] = p.load(trees[k])
        torch.cuda.synchronize()
        for g, s in zip(graphs, streams):
            with torch.cuda.stream(s):
                g.replay()
        torch.cuda.synchronize()
        for k, p in enumerate(ps):
            turned_rows(p, 63)
            check_step(p, hosts[k], trees[k], held[k], base[k])

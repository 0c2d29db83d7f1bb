"""Drafted decoding and rotary positions on the CPU: the entry points are exported, and every
refusal comes before any HIP call."""
import ctypes
import math
import os
import re

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

ce = pytest.importorskip("paper_2608_29291_amd")
torch = pytest.importorskip("torch")

FAKE = 0x10000  # never dereferenced: validation fails first
INV, UNS, WS = -1, -2, -3


@pytest.mark.parametrize("header,names", [
    ("ce_router_draft.h", ["ce_draft_masks", "ce_kv_keep", "ce_kv_trim", "ce_paged_tree_attention", "ce_verify_drafts",
                           "ce_verify_workspace_size"]),
    ("ce_router_rotary.h", ["ce_rotary"])])
def test_every_declared_symbol_is_exported(header, names):
    txt = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", header)).read(), flags=re.S)
    assert sorted(set(re.findall(r"\b(ce_[a-z_]+)\s*\(", txt))) == names
    for n in names:
        assert hasattr(ce.lib, n), n


def drafts(**kw):
    d = ce.CEDrafts(4, 20, FAKE, FAKE, FAKE)
    for k, v in kw.items():
        setattr(d, k, v)
    return d


def cache(**kw):
    c = ce.CEKVCache(4, 2, 128, 16, 100, 10, ce.CE_BF16, 2 * 16 * 128, FAKE, FAKE, None, None, FAKE)
    for k, v in kw.items():
        setattr(c, k, v)
    return c


def attn(**kw):
    a = ce.CEPagedAttn(12, 64, FAKE, FAKE, 0, 0.1)
    for k, v in kw.items():
        setattr(a, k, v)
    return a


def masks(d, words=2, mask=FAKE):
    return ce.lib.ce_draft_masks(None if d is None else ctypes.byref(d), words, None, mask, None, None, None)


def attend(c, a, mask=FAKE, words=2, q=FAKE, ld=12 * 128, o=FAKE, ws=FAKE, ws_bytes=1 << 40):
    return ce.lib.ce_paged_tree_attention(ctypes.byref(c), ctypes.byref(a), mask, words, q, ld, o, ws, ws_bytes, None)


def verify(d, vocab=1000, logits=FAKE, ld=1000, dtype=ce.CE_BF16, probs=FAKE, pld=1000, ua=FAKE, us=FAKE, kept=FAKE, n=FAKE,
           nxt=FAKE, ws=FAKE & ~255, ws_bytes=1 << 40):
    return ce.lib.ce_verify_drafts(None if d is None else ctypes.byref(d), vocab, logits, ld, dtype, None, probs, pld, ua, us,
                                   kept, n, nxt, ws, ws_bytes, None)


def size(d, vocab=1000, probs=1):
    return ce.lib.ce_verify_workspace_size(None if d is None else ctypes.byref(d), vocab, probs)


def keep(c, rows=8, off=FAKE, start=FAKE, kept=FAKE, n=FAKE):
    return ce.lib.ce_kv_keep(None if c is None else ctypes.byref(c), off, rows, start, kept, n, None)


def trim(c, **null):
    p = [None if n in null else FAKE for n in ("lens", "start", "n_kept", "free", "count", "lens_out", "count_out")]
    return ce.lib.ce_kv_trim(None if c is None else ctypes.byref(c), *p, None, None)


@pytest.mark.parametrize("kw,code", [({"B": 0}, INV), ({"row_capacity": -1}, INV), ({"B": 65536}, UNS),
                                     ({"row_capacity": 1 << 24}, UNS)])
def test_tree_sizes(kw, code):
    d = drafts(**kw)
    assert masks(d) == verify(d) == code
    assert size(d) == 0


def test_masks_refusals():
    assert masks(None) == masks(drafts(offsets=None)) == masks(drafts(), words=0) == INV
    assert masks(drafts(), words=65) == UNS
    assert masks(drafts(), mask=None) == 0  # nothing is asked for


def test_tree_attention_refusals():
    assert attend(cache(), attn(), mask=None) == attend(cache(), attn(), words=0) == attend(cache(), attn(causal=1)) == INV
    assert attend(cache(), attn(), words=65) == UNS
    assert attend(cache(), attn(), ld=12 * 128 - 8) == attend(cache(), attn(), q=None) == INV
    assert attend(cache(head_dim=64), attn()) == attend(cache(), attn(q_capacity=1 << 26)) == UNS
    assert attend(cache(max_pages=1000), attn(), ws=None) == WS
    assert attend(cache(), attn(q_capacity=0), q=None, o=None, ws=None, ws_bytes=0) == 0


def test_verify_refusals():
    d = drafts()
    assert verify(None) == verify(drafts(offsets=None)) == verify(drafts(tokens=None)) == INV
    for kw in ({"vocab": 0}, {"ld": 999}, {"pld": 999}, {"logits": None}, {"us": None}, {"kept": None}, {"n": None},
               {"nxt": None}, {"ua": None}, {"probs": None}):
        assert verify(d, **kw) == INV, kw
    for kw in ({"vocab": 1 << 24, "ld": 1 << 24, "pld": 1 << 24}, {"dtype": ce.CE_E4M3}, {"ld": 1 << 32}, {"pld": 1 << 32}):
        assert verify(d, **kw) == UNS, kw
    assert verify(drafts(row_capacity=(1 << 24) - 1), vocab=1 << 17, ld=1 << 17, pld=1 << 17) == UNS
    big = dict(vocab=1100000, ld=1100000, pld=1100000)  # (more workgroups than a launch may have)
    assert verify(drafts(B=65535), **big) == UNS and size(drafts(B=65535), vocab=1100000) == 0
    need = size(d)
    assert 0 < size(d, probs=0) < need
    assert verify(d, ws=None) == verify(d, ws=FAKE + 16) == verify(d, ws_bytes=need - 1) == WS
    assert size(None) == size(d, vocab=0) == size(drafts(row_capacity=0)) == 0


def test_keep_and_trim_refusals():
    for kw, code in (({"B": 0}, INV), ({"page_size": 24}, UNS), ({"n_pages": 0}, INV), ({"max_pages": (1 << 26) + 1}, UNS)):
        assert keep(cache(**kw)) == trim(cache(**kw)) == code
    assert keep(cache(head_dim=64)) == UNS and keep(cache(page_stride=16)) == INV
    assert keep(None) == trim(None) == keep(cache(), rows=-1) == INV
    assert keep(cache(), rows=1 << 24) == UNS
    for kw in ({"off": None}, {"start": None}, {"kept": None}, {"n": None}):
        assert keep(cache(), **kw) == INV, kw
    assert keep(cache(k=None)) == keep(cache(page_table=None)) == trim(cache(page_table=None)) == INV
    for n in ("lens", "start", "n_kept", "free", "count", "lens_out", "count_out"):
        assert trim(cache(), **{n: True}) == INV, n
    assert keep(cache(), rows=0, kept=None) == 0  # nothing to do is no launch


def rotary(freqs=(1.0,) * 32, axes=None, x=FAKE, ld=1024, y=FAKE, yld=1024, positions=FAKE, **kw):
    f = None if freqs is None else (ctypes.c_double * len(freqs))(*freqs)
    a = None if axes is None else (ctypes.c_int32 * len(axes))(*axes)
    d = ce.CERotaryDesc(10, 8, 128, 32, 2, 0, 0, ce.CE_BF16, 100, ctypes.cast(f, ctypes.c_void_p) if f else None,
                        ctypes.cast(a, ctypes.c_void_p) if a else None, positions, None)
    for k, v in kw.items():
        setattr(d, k, v)
    return ce.lib.ce_rotary(ctypes.byref(d), x, ld, y, yld, None)


def test_rotary_refusals():
    assert ce.lib.ce_rotary(None, FAKE, 1024, FAKE, 1024, None) == INV
    for kw in ({"rows": -1}, {"n_heads": 0}, {"head_dim": 0}, {"n_pairs": 0}, {"n_axes": 0}, {"n_positions": -1},
               {"layout": 2}, {"inverse": 2}, {"freqs": None}, {"x": None}, {"y": None}, {"positions": None}, {"ld": 1016},
               {"yld": 1020}, {"ld": 1032}, {"freqs": [math.nan] * 32}, {"freqs": [65.0] * 32}, {"axes": [0] * 31 + [2]},
               {"axes": [-1] * 32}):
        assert rotary(**kw) == INV, kw
    for kw in ({"head_dim": 258}, {"head_dim": 129}, {"n_pairs": 65}, {"n_axes": 5}, {"dtype": ce.CE_E4M3}, {"n_heads": 1 << 16},
               {"rows": 1 << 30}):
        assert rotary(**kw) == UNS, kw
    assert rotary(rows=1 << 25, n_heads=1, head_dim=256, n_pairs=1, freqs=[1.0], y=2 * FAKE) == UNS
    assert rotary(rows=0, x=None, y=None) == 0


def test_binding_refuses_what_a_pointer_cannot_say():
    i = torch.zeros(3, dtype=torch.int32)
    f = torch.zeros(3, 10)
    x = torch.zeros(3, 2, 128)
    d = ce.Drafts(i, i, i)
    for call in (lambda: ce.ce_draft_masks(d, torch.zeros(3, 1, dtype=torch.int32)), lambda: ce.Drafts(i).c(),
                 lambda: ce.Drafts(None, i).c(), lambda: ce.ce_verify_drafts(d, f, i, i, i, i),
                 lambda: ce.Rotary([1.0], [0, 0]), lambda: ce.ce_rotary(ce.Rotary([1.0]), x, x, i),
                 lambda: ce.ce_rotary(ce.Rotary([1.0]), x, x[:2], i),
                 lambda: ce.ce_kv_keep(ce.KVCache(x, x, i), i, i, i, i)):
        with pytest.raises(ValueError):
            call()

"""The paged cache on the CPU: its entry points are exported, and every refusal
comes before any HIP call."""
import ctypes
import os
import re

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HEADER = os.path.join(ROOT, "include", "ce_router_paged.h")

ce = pytest.importorskip("paper_2608_29291_amd")
torch = pytest.importorskip("torch")

FAKE = 0x10000  # never dereferenced: validation fails first


def test_every_declared_symbol_is_exported():
    txt = re.sub(r"/\*.*?\*/", "", open(HEADER).read(), flags=re.S)
    names = sorted(set(re.findall(r"\b(ce_[a-z_]+)\s*\(", txt)))
    assert names == ["ce_kv_append", "ce_kv_reserve", "ce_paged_attention", "ce_paged_workspace_size"]
    for n in names:
        assert hasattr(ce.lib, n), n


def cache(**kw):
    c = ce.CEKVCache(4, 2, 128, 16, 100, 10, ce.CE_BF16, 2 * 16 * 128, FAKE, FAKE, None, None, FAKE)
    for k, v in kw.items():
        setattr(c, k, v)
    return c


def attn(**kw):
    a = ce.CEPagedAttn(12, 64, FAKE, FAKE, 1, 0.1)
    for k, v in kw.items():
        setattr(a, k, v)
    return a


INV, UNS, WS = -1, -2, -3
TABLE = [({"B": 0}, INV), ({"page_size": 0}, INV), ({"n_pages": 0}, INV), ({"max_pages": 0}, INV), ({"B": 65536}, UNS),
         ({"page_size": 8}, UNS), ({"page_size": 48}, UNS), ({"page_size": 512}, UNS), ({"n_pages": 1 << 27}, UNS),
         ({"max_pages": (1 << 26) + 1}, UNS)]
PAGES = [({"n_kv_heads": 0}, INV), ({"head_dim": 64}, UNS), ({"dtype": ce.CE_F32}, UNS), ({"dtype": 3}, UNS),
         ({"page_stride": 2 * 16 * 128 - 16}, INV), ({"page_stride": 2 * 16 * 128 + 8}, INV),
         ({"page_stride": 1 << 31}, UNS), ({"k_scale": FAKE}, INV), ({"k_scale": FAKE, "v_scale": FAKE}, INV),
         ({"dtype": ce.CE_E4M3, "v_scale": FAKE}, INV), ({"n_kv_heads": 1 << 16, "page_stride": 1 << 28}, UNS)]
ATTN = [({"n_heads": 0}, INV), ({"n_heads": 13}, INV), ({"q_capacity": -1}, INV), ({"causal": 2}, INV),
        ({"scale": 0.0}, INV), ({"scale": -1.0}, INV), ({"scale": float("nan")}, INV), ({"scale": float("inf")}, INV),
        ({"scale": 3e38}, INV), ({"n_heads": 2 * 4097}, UNS),
        ({"q_capacity": 1 << 26}, UNS)]


def reserve(c, rows=8, new=FAKE, **null):
    names = ["lens", "free", "count", "lens_out", "count_out", "start", "slots"]
    p = {n: None if n in null else FAKE for n in names}
    return ce.lib.ce_kv_reserve(None if c is None else ctypes.byref(c), p["lens"], new, rows, None, p["free"], p["count"],
                                p["lens_out"], p["count_out"], p["start"], p["slots"], None, None)


def append(c, rows=8, k=FAKE, v=FAKE, slots=FAKE, kld=256, vld=256):
    return ce.lib.ce_kv_append(None if c is None else ctypes.byref(c), k, kld, v, vld, slots, rows, None)


def attend(c, a, q=FAKE, ld=12 * 128, o=FAKE, ws=FAKE, ws_bytes=1 << 40):
    return ce.lib.ce_paged_attention(None if c is None else ctypes.byref(c), None if a is None else ctypes.byref(a), q, ld,
                                     o, ws, ws_bytes, None)


def size(c, a):
    return ce.lib.ce_paged_workspace_size(None if c is None else ctypes.byref(c), None if a is None else ctypes.byref(a))


@pytest.mark.parametrize("kw,code", TABLE)
def test_table_sizes(kw, code):
    c = cache(**kw)
    assert reserve(c) == append(c) == attend(c, attn()) == code
    assert size(c, attn()) == 0


@pytest.mark.parametrize("kw,code", PAGES)
def test_page_sizes(kw, code):
    c = cache(**kw)
    assert append(c) == attend(c, attn()) == code
    assert size(c, attn()) == 0


@pytest.mark.parametrize("kw,code", ATTN)
def test_attention_sizes(kw, code):
    assert attend(cache(), attn(**kw)) == code
    assert size(cache(), attn(**kw)) == 0


def test_null_pointers():
    assert reserve(None) == append(None) == attend(None, attn()) == attend(cache(), None) == INV
    for n in ("lens", "free", "count", "lens_out", "count_out", "start", "slots"):
        assert reserve(cache(), **{n: True}) == INV, n
    assert reserve(cache(page_table=None)) == INV
    assert reserve(cache(), rows=-1) == INV and reserve(cache(), new=None) == INV
    for kw in ({"k": None}, {"v": None}, {"slots": None}):
        assert append(cache(), **kw) == INV
    assert append(cache(k=None)) == append(cache(v=None)) == INV
    assert attend(cache(k=None), attn()) == attend(cache(page_table=None), attn()) == INV
    for kw in ({"q": None}, {"o": None}):
        assert attend(cache(), attn(), **kw) == INV
    assert attend(cache(), attn(q_offsets=None)) == attend(cache(), attn(lens=None)) == INV


def test_row_strides():
    assert append(cache(), kld=255) == append(cache(), vld=252) == append(cache(), kld=128) == INV
    assert append(cache(), kld=1 << 31) == append(cache(), vld=1 << 31) == UNS
    assert attend(cache(), attn(), ld=12 * 128 - 8) == attend(cache(), attn(), ld=12 * 128 + 4) == INV
    assert attend(cache(), attn(), ld=1 << 22) == UNS


def test_workspace():
    c, a = cache(max_pages=1000), attn()
    need = size(c, a)
    assert 0 < need <= 35 << 20
    assert attend(c, a, ws=None) == attend(c, a, ws_bytes=need - 1) == attend(c, a, ws=FAKE + 16) == WS
    # short sequences are never cut; more than 256 are planned in memory; no rows need nothing
    assert size(cache(max_pages=15), a) == 0
    assert 0 < size(cache(max_pages=15, B=300), a) <= 8192
    assert size(c, attn(q_capacity=0)) == 0
    for B in (1, 256, 257, 65535):
        for hkv in (1, 2, 4, 60):
            for rows in (1, 64, 1 << 20):
                cc = cache(B=B, n_kv_heads=hkv, page_stride=hkv * 2048, max_pages=1 << 20)
                assert size(cc, attn(n_heads=hkv * 2, q_capacity=rows)) <= 35 << 20
    assert size(cache(B=65535, n_kv_heads=65, page_stride=65 * 2048), attn(n_heads=65)) == 0  # refused


def test_workspace_for_more_rows_serves_fewer():
    for B in (4, 40, 300):
        for heads in (2, 12, 64):
            sizes = [size(cache(max_pages=1000, B=B), attn(n_heads=heads, q_capacity=n)) for n in range(1, 700, 7)]
            assert sizes == sorted(sizes)


def test_nothing_to_do_is_no_launch():
    assert append(cache(), rows=0, k=None, v=None, slots=None) == 0
    assert attend(cache(), attn(q_capacity=0), q=None, o=None, ws=None, ws_bytes=0) == 0


def test_binding_refuses_what_a_pointer_cannot_say():
    k = torch.zeros(4, 2, 16, 128, dtype=torch.bfloat16)
    t = torch.zeros(3, 5, dtype=torch.int32)
    i = torch.zeros(3, dtype=torch.int32)
    for c in (ce.KVCache(k, k, t), ce.KVCache(k[0], k[0], t), ce.KVCache(k, k[:2], t), ce.KVCache(k, k, t[0]),
              ce.KVCache(None, k, t), ce.KVCache(k.float(), k.float(), t)):
        for call in (lambda: ce.ce_kv_reserve(c, i, None, i, i, i, None),
                     lambda: ce.ce_kv_append(c, k[0], k[0], i),
                     lambda: ce.ce_paged_attention(c, k[0], k[0], i, i, True, 1.0),
                     lambda: ce.ce_paged_workspace_size(c, 1, 2)):
            with pytest.raises(ValueError):
                call()

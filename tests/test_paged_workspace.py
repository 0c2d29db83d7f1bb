"""The bound that the header gives for the workspace of paged attention."""
import ctypes
import os
import re

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

ce = pytest.importorskip("paper_2608_29291_amd")

FAKE = 0x10000  # never dereferenced: sizes only


def test_the_bound_is_reached_and_not_passed():
    text = open(os.path.join(ROOT, "include", "ce_router_paged.h")).read()
    bound = int(re.search(r"is at most (\d+) bytes", text).group(1))
    most = 0
    for B in (1, 256, 257, 65534, 65535):
        for hkv in (1, 2, 64):
            for g in (1, 8, 9, 4096):
                for rows in (1, B - 1, B, B + 1, 1 << 20, 1 << 27):
                    for page, pages in ((16, 10), (16, 1000), (256, 1 << 22)):
                        c = ce.CEKVCache(B, hkv, 128, page, 100, pages, ce.CE_BF16, hkv * page * 128, FAKE, FAKE, None, None, FAKE)
                        a = ce.CEPagedAttn(hkv * g, rows, FAKE, FAKE, 1, 0.1)
                        most = max(most, ce.lib.ce_paged_workspace_size(ctypes.byref(c), ctypes.byref(a)))
    assert most == bound

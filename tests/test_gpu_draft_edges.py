"""Drafted decoding where its arguments end: offsets out of order, long sequences, large batches."""
import numpy as np
import pytest
import torch

import draft_util as du
from test_gpu_verify import Case

pytestmark = pytest.mark.gpu
ce = pytest.importorskip("paper_2608_29291_amd")


@pytest.mark.parametrize("drawn", [False, True])
@pytest.mark.parametrize("off", [[0, 25, 5, 30], [-3, 10, 20, 1 << 30], [7, 7, 7, 7], [30, 20, 10, 0], [0, 30, 10, 30]])
def test_every_sequence_gets_a_count_and_a_token_whatever_the_offsets(off, drawn):
    # the calls behind this one take lengths from the count: it must not be what the memory held before
    c = Case([10, 10, 10], 500, torch.float32, drawn=drawn)
    c.off = np.array(off, np.int32)
    for pad in (3, 5000):
        for fill in (0xff, 0):
            _, n_kept, following = c.run(rest=False, pad=pad, fill=fill)  # (filled with -9 before)
            assert all(0 <= k <= 30 + pad for k in n_kept), n_kept
            assert all(-1 <= t < 500 for t in following), following
            ends = np.clip(c.off, 0, 30 + pad)
            assert all(k == 0 and t == -1 for k, t, lo, hi in zip(n_kept, following, ends, ends[1:]) if hi <= lo)

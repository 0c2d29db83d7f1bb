"""Values at the ends of their range in attention over the paged cache: infinite scores beside
finite rows."""
import numpy as np
import pytest

import paged_util as U

pytestmark = pytest.mark.gpu

SHAPES = [([1, 1], [900, 40]), ([3, 2], [900, 40]), ([150, 40], [1500, 64])]  # single tokens, few rows, tiles


def rows(n, heads, seed=1):
    return U.bf16(np.random.default_rng(seed).standard_normal((n, heads, U.DH)))


def go(p, q, new, scale=U.DH ** -0.5):
    """Outputs of rows q, causal."""
    import torch
    import paper_2608_29291_amd as ce
    qd = torch.from_numpy(q).to(torch.bfloat16).cuda()
    o = torch.full_like(qd, 77.0)
    i32 = lambda x: torch.tensor(x, dtype=torch.int32).cuda()
    ce.ce_paged_attention(p.cache(), qd, o, i32([0] + np.cumsum(new).tolist()), i32(p.lens), True, scale)
    return o.float().cpu().numpy()


@pytest.mark.parametrize("new,lens", SHAPES[1:])
def test_infinite_scores_touch_the_rows_that_see_them(new, lens):
    """Keys of -infinity weigh nothing, a whole chunk of them too. A key of +infinity near the
    end makes NaN of the rows that see it; earlier rows, other heads and the next sequence
    stay finite."""
    p = U.Paged(lens, 2, 16, "bf16", seed=21)
    k = [x.copy() for x in p.k]
    k[0][:700, 0, 0] = -np.inf
    k[0][lens[0] - new[0] + new[0] // 2, 1, 0] = np.inf
    p = U.Paged(lens, 2, 16, "bf16", seed=21, k=k)
    q = rows(sum(new), 12)
    q[:, :, 0] = np.abs(q[:, :, 0]) + 0.5
    q[0, 1, 0] = -1.0  # +infinity from the first key on
    want, top = p.answer(q, new, True, U.DH ** -0.5)
    bad = np.isnan(want).all(2)
    for r in range(sum(new)):
        assert bad[r].tolist() == [(h == 1 and r == 0) or (h >= 6 and new[0] // 2 <= r < new[0]) for h in range(12)]
    U.check(go(p, q, new), want, top)

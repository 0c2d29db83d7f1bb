"""Routed attention with scores so large that one key has all the weight: prefill, bidirectional
and decode rows against the float64 oracle.

Tolerance. The weight of that key is 1 and the others' are 0, exactly, so the output is its value,
a bf16 number: half a step of it (2^-8) is allowed. Compared are the rows whose highest score
leads by more than 2^-12 of its size; a fp32 sum of 128 products errs by about 2^-16 of it."""
import numpy as np
import pytest

from ce_workloads import make_attention_inputs
from oracle import attention as oa

pytestmark = pytest.mark.gpu

DH = 128


def to_bf16(x):
    import torch
    return torch.from_numpy(np.asarray(x, np.float32)).to(torch.bfloat16)


@pytest.mark.parametrize("size,scale", [(3e3, 0.1), (3e4, 0.1), (1e6, 0.1), (1e9, 0.1), (1e18, 100.0)])
@pytest.mark.parametrize("q_lens,kv_lens,H,Hkv,causal", [([130, 40], [300, 40], 12, 2, True), ([200], [300], 4, 4, False),
                                                         ([1, 1, 1], [3000, 700, 65], 28, 4, True)])
def test_scores_of_any_size(q_lens, kv_lens, H, Hkv, causal, size, scale):
    import torch
    import paper_2608_29291_amd as ce
    q, k, v, qo, ko = make_attention_inputs(q_lens, kv_lens, H, Hkv, DH, seed=H)
    dq, dk, dv = to_bf16(q * size).cuda(), to_bf16(k * size).cuda(), to_bf16(v).cuda()
    q, k, v = (x.float().cpu().numpy().astype(np.float64) for x in (dq, dk, dv))
    want = oa.attention(q, k, v, qo, ko, Hkv, causal, float(np.float32(scale)))
    sure = np.zeros(q.shape[:2], bool)
    for b, (n, m) in enumerate(zip(q_lens, kv_lens)):
        for i in range(n):
            sees = m - n + i + 1 if causal else m
            for h in range(H):
                s = np.sort(k[ko[b]:ko[b] + sees, h // (H // Hkv)] @ q[qo[b] + i, h])
                sure[qo[b] + i, h] = len(s) < 2 or s[-1] - s[-2] > 2.0 ** -12 * np.abs(s).max()
    assert sure.mean() > 0.97
    o = torch.full(dq.shape, float("nan"), dtype=torch.bfloat16, device="cuda")
    up = lambda x: torch.from_numpy(np.asarray(x, np.int32)).cuda()
    ce.ce_routed_attention(dq, dk, dv, o, up(qo), up(ko), causal, scale)
    got = o.float().cpu().numpy()
    assert np.isfinite(got).all()
    assert (np.abs(got - want) <= 2.0 ** -8 * np.abs(want))[sure].all()

"""Batches of more sequences than a wave has lanes: work is found group by group, whatever the order of lengths."""

import numpy as np
import pytest
import torch

import attn_oracle as ao
from paper_2605_07238_amd import fate
from test_gpu_attention import BF, HF, compare, make_paged, run_paged

pytestmark = pytest.mark.gpu


def lengths(B, seed):
    rng = np.random.default_rng(seed)
    new = rng.integers(0, 9, B)
    kv = new + rng.integers(0, 70, B) * (rng.random(B) < 0.8)
    kv[B // 3], kv[B - 2] = 1500, 2300  # long ones in the first and in the last group
    new[B - 2] = 40
    new[5], kv[5] = 3, 0
    return new.tolist(), kv.tolist()


@pytest.mark.parametrize("B", [64, 65, 150, 400])
@pytest.mark.parametrize("most", [8, None])
def test_paged(B, most):
    new, kv = lengths(B, B)
    if most:
        new = [min(n, most) for n in new]
    args = make_paged(new, kv, 4, 2, 64, HF, 8, seed=B)
    want = ao.paged(*args[:3], args[3].tolist(), args[4].tolist(), args[5].tolist(), 0.125)
    status = torch.zeros(B, dtype=torch.int32, device="cuda")
    compare(*run_paged(*args, max_new=most, scale=0.125, status=status), want)
    assert not status.any()
    kv2 = args[4].copy()
    kv2[B - 1] = -1
    run_paged(*args[:4], kv2, args[5], max_new=most, status=status)
    assert status.tolist() == [0] * (B - 1) + [fate.FATE_EINVAL]


@pytest.mark.parametrize("B", [64, 65, 200])
def test_prompt(B):
    rng = np.random.default_rng(B)
    lens = rng.integers(0, 40, B)
    lens[B - 1], lens[3] = 300, 200
    off = np.concatenate([[0], np.cumsum(lens)]).astype(np.int32)
    gen = torch.Generator().manual_seed(B)
    q, k, v = (torch.randn(int(off[-1]), h, 64, generator=gen).to(BF) for h in (4, 2, 2))
    status = torch.zeros(B, dtype=torch.int32, device="cuda")
    out, lse = fate.fate_attn_prompt(q.cuda(), k.cuda(), v.cuda(), torch.from_numpy(off).cuda(), lse=True, status=status)
    compare(out, lse, ao.prompt(q, k, v, off.tolist(), 0.125))
    assert not status.any()
    bad = off.copy()
    bad[B] += 1
    fate.fate_attn_prompt(q.cuda(), k.cuda(), v.cuda(), torch.from_numpy(bad).cuda(), status=status)
    assert status.tolist() == [0] * (B - 1) + [fate.FATE_EINVAL]

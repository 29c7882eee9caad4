"""Offsets and lengths of a call's sequences: rows outside every sequence are no error of any, and what is an error in the
attention calls is one in the append."""

import math

import numpy as np
import pytest
import torch

from paper_2605_07238_amd import fate
from test_gpu_attention import HF

pytestmark = pytest.mark.gpu
BAD = fate.FATE_EINVAL


def ints(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def append(qkv, hq, hkv, cache, off, kv, pages, q_out):
    """The append of a fused projection; returns the status."""
    status = torch.zeros(len(kv), dtype=torch.int32, device="cuda")
    table = fate.rotation_table(256, 64)
    fate.fate_kv_append(qkv[:, :hq], qkv[:, hq:hq + hkv], qkv[:, hq + hkv:], *cache, ints(off), ints(kv), ints(pages), table,
                        q_out=q_out, status=status)
    return status.tolist()


def empty_cache(pages=40):
    return [torch.zeros(pages, 2, 16, 64, dtype=HF, device="cuda") for _ in range(2)]


@pytest.mark.parametrize("new,kv", [([3, 0, 40], [20, 0, 70]), ([0, 5], [0, 9]), ([1], [1]), ([1] * 70, [2] * 70)])
@pytest.mark.parametrize("lead,trail", [(5, 9), (5, 0), (0, 9), (2000, 3)])
def test_append_leaves_rows_outside_sequences_alone(new, kv, lead, trail):
    gen = torch.Generator(device="cuda").manual_seed(lead)
    T, need = sum(new), [-(-n // 16) for n in kv]
    off = np.concatenate([[0], np.cumsum(new)])
    at = np.concatenate([[0], np.cumsum(need)])
    pages = [[*range(at[b], at[b + 1])] + [-1] * (max(need) - need[b]) for b in range(len(new))]
    qkv = torch.randn(T, 8, 64, generator=gen, device="cuda").half()
    want, want_q = empty_cache(at[-1] + 1), torch.empty(T, 4, 64, dtype=HF, device="cuda")
    assert append(qkv, 4, 2, want, off, kv, pages, want_q) == [0] * len(new)
    padded = torch.full((lead + T + trail, 8, 64), math.nan, dtype=HF, device="cuda")
    padded[lead:lead + T] = qkv
    got, got_q = empty_cache(at[-1] + 1), torch.full((lead + T + trail, 4, 64), 3.0, dtype=HF, device="cuda")
    assert append(padded, 4, 2, got, off + lead, kv, pages, got_q) == [0] * len(new)
    assert torch.equal(got_q[lead:lead + T], want_q)
    assert (got_q[:lead] == 3).all() and (got_q[lead + T:] == 3).all()
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


@pytest.mark.parametrize("what", [-1, 33])
@pytest.mark.parametrize("B", [3, 90])
def test_append_reports_what_attention_reports(what, B):
    """A length out of range on a sequence with no tokens in the call."""
    off, kv, pages = [0] + [2] * (B - 1) + [5], [2] + [0] * (B - 2) + [7], [[0, 1]] + [[-1, -1]] * (B - 2) + [[2, 3]]
    kv[B - 2] = what
    qkv = torch.randn(5, 8, 64, device="cuda").half()
    cache = empty_cache()
    want = [BAD if b == B - 2 else 0 for b in range(B)]
    q = torch.empty(5, 4, 64, dtype=HF, device="cuda")
    assert append(qkv, 4, 2, cache, off, kv, pages, q) == want
    assert torch.equal(cache[1][0, :, :2], qkv[:2, 6:].transpose(0, 1)) and cache[1][2, :, 4:7].any()
    for most in (3, None):
        status = torch.zeros(B, dtype=torch.int32, device="cuda")
        fate.fate_attn_paged(q, *cache, ints(off), ints(kv), ints(pages), max_new=most, status=status)
        assert status.tolist() == want

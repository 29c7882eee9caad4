"""Offsets that are sound but leave rows outside, and offsets, lengths and empty sequences that are not sound: all calls
that read them hold the same ones for errors, report each, and leave the others' results as they are."""

import math

import numpy as np
import pytest
import torch

import attn_oracle as ao
from paper_2605_07238_amd import fate
from test_gpu_attention import BF, HF, compare, run_paged

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


def ascending_up_to(off, T):
    """The sequences that are sound: within the rows, not descending, not from below an earlier entry."""
    return [0 <= off[b] <= off[b + 1] <= T and off[b] >= max(off[:b + 1]) for b in range(len(off) - 1)]


OFFSETS = {
    "down": ([0, 10, 5, 20], 20),
    "twice the same rows": ([0, 20, 0, 20], 20),
    "first": ([6, 2, 20], 20),
    "past the end": ([0, 8, 40, 12, 20], 20),
    "negative": ([-3, 4, 20], 20),
    "down in a later group": ([*range(70), 20, *range(71, 131)], 130),
    "over a whole group": ([0, 1, 2, 100, *range(4, 131)], 130),
    "many times the same rows": ([0, 130] * 60, 130),
}


@pytest.mark.parametrize("name", sorted(OFFSETS))
def test_offsets_that_descend(name):
    off, T = OFFSETS[name]
    B = len(off) - 1
    good = ascending_up_to(off, T)
    want = [0 if x else BAD for x in good]
    kv = [140 if b % 3 else 131 for b in range(B)]
    P, need = 16, 9
    gen = torch.Generator().manual_seed(B)
    rng = np.random.default_rng(B)
    pages = rng.permutation(B * need).reshape(B, need).astype(np.int32)
    q = torch.randn(T, 4, 64, generator=gen).to(BF)
    kc, vc = (torch.randn(B * need, 2, P, 64, generator=gen).to(BF) for _ in range(2))
    for most in (4, None):
        status = torch.zeros(B, dtype=torch.int32, device="cuda")
        out, lse = run_paged(q, kc, vc, np.array(off, np.int32), np.array(kv, np.int32), pages, max_new=most, scale=0.125,
                             status=status)
        assert status.tolist() == want
        for b in range(B):
            if good[b] and off[b] < off[b + 1]:
                lo, hi = off[b], off[b + 1]
                ref = ao.paged(q[lo:hi], kc, vc, [0, hi - lo], [kv[b]], [pages[b].tolist()], 0.125)
                compare(out[lo:hi], lse[lo:hi], ref)
    k, v = (torch.randn(T, 2, 64, generator=gen).to(BF) for _ in range(2))
    status.zero_()
    out, lse = fate.fate_attn_prompt(q.cuda(), k.cuda(), v.cuda(), ints(off), lse=True, status=status)
    assert status.tolist() == want
    for b in range(B):
        if good[b] and off[b] < off[b + 1]:
            rows = slice(off[b], off[b + 1])
            compare(out[rows], lse[rows], ao.prompt(q[rows], k[rows], v[rows], [0, off[b + 1] - off[b]], 0.125))
    # append: rows of sound sequences are stored, no others are
    nk, nv = torch.zeros_like(kc).cuda(), torch.zeros_like(vc).cuda()
    status.zero_()
    fate.fate_kv_append(None, k.cuda(), v.cuda(), nk, nv, ints(off), ints(kv), torch.from_numpy(pages).cuda(), status=status)
    assert status.tolist() == want
    ek, ev = torch.zeros_like(kc), torch.zeros_like(vc)
    for b in range(B):
        if good[b]:
            for t in range(off[b], off[b + 1]):
                pos = kv[b] - off[b + 1] + t
                ek[pages[b, pos // P], :, pos % P], ev[pages[b, pos // P], :, pos % P] = k[t], v[t]
    assert torch.equal(nk.cpu(), ek) and torch.equal(nv.cpu(), ev)

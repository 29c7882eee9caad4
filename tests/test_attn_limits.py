"""Sizes that the attention entries cannot launch: refused as such on the host, before anything reaches a GPU."""

import ctypes as C

import pytest

from paper_2605_07238_amd import fate
from test_attn_entries import append, cache, heads, paged, prompt, rows, seqs

EINVAL, ERANGE = -1, -2


@pytest.mark.parametrize("T", [1 << 31, 1 << 54, 1 << 60, (1 << 63) - 1, (1 << 62) + 3])
def test_rows_past_any_count(T):
    """Products of T and heads that would pass 64 bits."""
    for f in (append, paged, prompt):
        assert f(s=seqs(T=T)) == ERANGE
    n = C.c_size_t(7)
    assert fate.load().fate_attn_paged_ws_size(heads(), seqs(T=T), cache(), 1, n) == ERANGE and n.value == 7


def test_grids_past_the_launch():
    """A launch takes fewer than 2^32 threads, in workgroups of 256.  What fits is shown by a later refusal: nothing here
    may reach a launch."""
    h, none = heads(heads_q=1, heads_kv=1), rows(data=None)
    most = (1 << 26) - 4  # an append takes four tokens a workgroup
    for T in (most + 1, 1 << 26, 1 << 29):
        assert append(h=h, s=seqs(T=T)) == append(h=h, s=seqs(T=T), k=none) == ERANGE
    assert append(h=h, s=seqs(T=most), k=none) == EINVAL
    # tiles: T G / 128 of them and one for each sequence, per key head
    h = heads(heads_q=32, heads_kv=32)
    n = C.c_size_t(7)
    for B, T, fits in ((600_000, 600_000, False), (1 << 19, 1 << 19, False), (1 << 18, 1 << 18, True), (1, 1 << 24, True),
                       (1 << 23, 1000, True)):
        want = EINVAL if fits else ERANGE
        assert prompt(h=h, s=seqs(B=B, T=T), k=none if fits else None) == want
        assert paged(h=h, s=seqs(B=B, T=T), most=min(T, 64), q=none if fits else None) == want
        assert fate.load().fate_attn_paged_ws_size(h, seqs(B=B, T=T), cache(), min(T, 64), n) == (0 if fits else ERANGE)
    # few new tokens a sequence: as many workgroups as run at once, whatever the batch
    assert paged(h=h, s=seqs(B=600_000, T=600_000), most=1, q=none) == EINVAL
    assert fate.load().fate_attn_paged_ws_size(h, seqs(B=600_000, T=600_000), cache(), 1, n) == 0


@pytest.mark.parametrize("heads_q,heads_kv,head_dim", [(64, 1, 64), (256, 1, 256), (32, 1, 128), (8, 8, 64), (20, 1, 256)])
def test_no_bound_below_one_token(heads_q, heads_kv, head_dim):
    """A call that has tokens is planned for one a sequence at least: the axis of work of few rows, its length in 64 bits,
    holds 2^31 rows over 2^30 keys only where a token has no more packed rows than a workgroup."""
    h = heads(heads_q=heads_q, heads_kv=heads_kv, head_dim=head_dim)
    c = cache(page=1024 * head_dim, head=16 * head_dim, token=head_dim)
    n = [C.c_size_t(0) for _ in range(2)]
    for most in (0, 1):
        assert fate.load().fate_attn_paged_ws_size(h, seqs(T=1000), c, most, n[most]) == 0
    assert n[0].value == n[1].value > 0

"""Sizes that the attention entries cannot launch: refused as such on the host, before anything reaches a GPU."""

import ctypes as C

import pytest

from paper_2605_07238_amd import fate
from test_attn_entries import append, cache, heads, paged, prompt, rows, seqs

ERANGE = -2


@pytest.mark.parametrize("T", [1 << 31, 1 << 54, 1 << 60, (1 << 63) - 1, (1 << 62) + 3])
def test_rows_past_any_count(T):
    """Products of T and heads that would pass 64 bits."""
    for f in (append, paged, prompt):
        assert f(s=seqs(T=T)) == ERANGE
    n = C.c_size_t(7)
    assert fate.load().fate_attn_paged_ws_size(heads(), seqs(T=T), cache(), 1, n) == ERANGE and n.value == 7

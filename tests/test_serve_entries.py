"""What the calls around a wave's attention refuse on the host, before anything reaches a GPU."""

import ctypes as C

import pytest

from paper_2605_07238_amd import fate
from test_attn_entries import cache, heads, rows, seqs

A = 1 << 20  # an aligned address that is never read
EINVAL, ERANGE = -1, -2


def kv_tables(**x):
    return fate.KvTables(**dict(dict(B=3, max_pages=4, page_size=16, n_pages=9, pages_stride=4, pages=A, free=A, n_free=A,
                                     kv_len=A), **x))


def reserve(t=None, new=A, T=7, off=A, kv=A, n=A, taken=A, slots=A, positions=A):
    return fate.load().fate_kv_reserve(t or kv_tables(), new, T, off, kv, n, taken, slots, positions, None, None)


def trim(t=None, keep=A, kv=A, n=A, given=A):
    return fate.load().fate_kv_trim(t or kv_tables(), keep, kv, n, given, None, None)


BAD_TABLES = [(dict(B=-1), EINVAL), (dict(max_pages=-1), EINVAL), (dict(n_pages=-1), EINVAL), (dict(pages_stride=-4), EINVAL),
              (dict(page_size=0), EINVAL), (dict(page_size=-16), EINVAL), (dict(page_size=24), EINVAL),
              (dict(page_size=2048), ERANGE), (dict(max_pages=1 << 27, pages_stride=1 << 27), ERANGE),
              (dict(B=(1 << 24) + 1), ERANGE), (dict(pages_stride=3), EINVAL), (dict(pages=None), EINVAL),
              (dict(pages=A + 2), EINVAL), (dict(free=None), EINVAL), (dict(n_free=None), EINVAL), (dict(n_free=A + 1), EINVAL),
              (dict(kv_len=None), EINVAL)]


@pytest.mark.parametrize("bad,status", BAD_TABLES, ids=str)
def test_tables(bad, status):
    for f in (reserve, trim):
        assert f(t=kv_tables(**bad)) == status


def test_reserve():
    assert fate.load().fate_kv_reserve(None, A, 7, A, A, A, A, A, A, None, None) == EINVAL
    assert reserve(T=-1) == EINVAL and reserve(T=1 << 31) == ERANGE and reserve(T=1 << 62) == ERANGE
    for name in ("new", "off", "kv", "n", "taken"):
        assert reserve(**{name: None}) == EINVAL and reserve(**{name: A + 2}) == EINVAL
    assert reserve(slots=A + 4) == EINVAL and reserve(positions=A + 2) == EINVAL


def test_trim():
    assert fate.load().fate_kv_trim(None, A, A, A, A, None, None) == EINVAL
    for name in ("keep", "kv", "n", "given"):
        assert trim(**{name: None}) == EINVAL and trim(**{name: A + 2}) == EINVAL


def test_axes():
    names = (C.c_uint8 * 32)(*([0] * 10 + [1] * 10 + [2] * 12))
    good = dict(n_axes=3, pair_axis=C.addressof(names), positions=A, stride=6)

    def append(rot=64, k="", **x):
        axes = fate.Axes(**dict(good, **x)) if x.get("n_axes", 1) is not None else None
        return fate.load().fate_kv_append_axes(heads(), seqs(), rows(), rows() if k == "" else k, rows(), A, 9, rot, 0, axes, cache(),
                                               rows(), None, None)

    for bad, status in ((dict(n_axes=None), EINVAL), (dict(n_axes=0), EINVAL), (dict(n_axes=2), EINVAL), (dict(n_axes=5), ERANGE),
                        (dict(pair_axis=None), EINVAL), (dict(positions=None), EINVAL), (dict(positions=A + 2), EINVAL),
                        (dict(stride=-1), EINVAL), (dict(rot=0), EINVAL), (dict(rot=63), EINVAL), (dict(k=None), EINVAL)):
        assert append(**bad) == status, bad
    assert fate.rotation_axes((2, 1, 3)) == (0, 0, 1, 2, 2, 2)
    assert fate.rotation_axes((2, 1, 3), cyclic=True) == (0, 1, 2, 0, 2, 2)
    assert fate.rotation_axes(()) == fate.rotation_axes((), cyclic=True) == ()


def test_shaped_scores():
    f = fate.load()

    def paged(scores, **x):
        return f.fate_attn_paged_shaped(heads(), seqs(), rows(), cache(), 2, 0.1, scores, rows(**x), None, None, A, 1 << 40, None)

    def prompt(scores, **x):
        return f.fate_attn_prompt_shaped(heads(), seqs(), rows(), rows(), rows(), 0.1, scores, rows(**x), None, None, None)

    for call in (paged, prompt):
        assert call(None) == EINVAL
        assert call(fate.Scores(), data=A + 8) == EINVAL  # as the plain calls check
        for bad in (dict(cap=-1.0), dict(cap=float("nan")), dict(cap=float("inf")), dict(cap=1e-44), dict(cap=3e38), dict(slopes=A + 2),
                    dict(prefix=A + 1), dict(start=A + 3)):
            assert call(fate.Scores(**bad)) == EINVAL, bad

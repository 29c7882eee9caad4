"""What the calls around a wave's attention refuse on the host, before anything reaches a GPU."""

import ctypes as C
import os
import subprocess

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


def sampling(**x):
    return fate.Sampling(**dict(dict(dtype=2, rows=3, vocab=100, stride=100, logits=A, u=A, temperature_all=1.0, top_p_all=1.0), **x))


def test_sampling():
    f, n = fate.load(), C.c_size_t(7)

    def call(s, token=A, logprob=A, status=A, ws=A, ws_bytes=1 << 40):
        return f.fate_sample(s, token, logprob, status, ws, ws_bytes, None)

    nan, inf = float("nan"), float("inf")
    for bad, status in ((dict(dtype=3), EINVAL), (dict(dtype=-1), EINVAL), (dict(rows=-1), EINVAL), (dict(vocab=0), EINVAL),
                        (dict(stride=-1), EINVAL), (dict(rows=1 << 22), ERANGE), (dict(vocab=(1 << 30) + 1), ERANGE),
                        (dict(temperature_all=-1.0), EINVAL), (dict(temperature_all=nan), EINVAL), (dict(temperature_all=inf), EINVAL),
                        (dict(top_k_all=-1), EINVAL), (dict(top_p_all=0.0), EINVAL), (dict(top_p_all=1.5), EINVAL),
                        (dict(top_p_all=nan), EINVAL), (dict(min_p_all=-0.5), EINVAL), (dict(min_p_all=1.5), EINVAL)):
        assert call(sampling(**bad)) == status, bad
        assert f.fate_sample_ws_size(sampling(**bad), n) == status and n.value == 7
    for bad in (dict(logits=None), dict(logits=A + 2), dict(logits=A + 1, dtype=0), dict(u=None), dict(u=A + 2), dict(temperature=A + 1),
                dict(top_k=A + 2), dict(top_p=A + 3), dict(min_p=A + 2)):
        assert call(sampling(**bad)) == EINVAL, bad
    assert call(None) == EINVAL and f.fate_sample_ws_size(None, n) == EINVAL and f.fate_sample_ws_size(sampling(), None) == EINVAL
    assert call(sampling(), token=None) == call(sampling(), token=A + 2) == call(sampling(), logprob=A + 2) == EINVAL
    assert call(sampling(), status=A + 2) == EINVAL
    assert call(sampling(rows=0, logits=None)) == 0


STRUCTS = [("fate_kv_tables_t", fate.KvTables), ("fate_axes_t", fate.Axes), ("fate_scores_t", fate.Scores), ("fate_sampling_t", fate.Sampling)]


def test_structs_as_the_header_has_them(tmp_path):
    lines, want = [], []
    for name, mirror in STRUCTS:
        lines.append('printf("%%zu\\n", sizeof(%s));' % name)
        want.append(C.sizeof(mirror))
        for field, _ in mirror._fields_:
            lines.append('printf("%%zu\\n", offsetof(%s, %s));' % (name, field))
            want.append(getattr(mirror, field).offset)
    (tmp_path / "a.c").write_text('#include <stddef.h>\n#include <stdio.h>\n#include "fate.h"\nint main(void) {\n%s\nreturn 0; }\n' % "\n".join(lines))
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    subprocess.run(["gcc", "-std=c11", "-I", os.path.join(root, "include"), str(tmp_path / "a.c"), "-o", str(tmp_path / "a")], check=True)
    out = subprocess.run([str(tmp_path / "a")], check=True, capture_output=True, text=True).stdout
    assert [int(x) for x in out.split()] == want

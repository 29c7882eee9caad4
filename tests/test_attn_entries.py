"""What the attention entries refuse on the host, before anything reaches a GPU."""

import ctypes as C
import os
import subprocess

import pytest

from paper_2605_07238_amd import fate

A = 1 << 20  # an aligned address that is never read


def heads(**x):
    return fate.Heads(**dict(dict(dtype=fate.FATE_BF16, heads_q=8, heads_kv=2, head_dim=64), **x))


def seqs(**x):
    return fate.Seqs(**dict(dict(B=2, max_pages=4, T=6, pages_stride=4, off=A, kv_len=A, pages=A), **x))


def rows(**x):
    return fate.Rows(**dict(dict(data=A, token=512, head=64), **x))


def cache(**x):
    return fate.KvCache(**dict(dict(k=A, v=A, page=2048, head=1024, token=64, n_pages=9, page_size=16), **x))


def append(h=None, s=None, q="", k="", v="", table=A, table_rows=9, rot=64, inter=0, c=None, qo=""):
    pick = lambda x, r: r if x == "" else x  # noqa: E731
    return fate.load().fate_kv_append(h or heads(), s or seqs(), pick(q, rows()), pick(k, rows()), pick(v, rows()), table,
                                      table_rows, rot, inter, c or cache(), pick(qo, rows()), None, None)


def paged(h=None, s=None, q=None, c=None, most=2, scale=0.1, out=None, ws=A, ws_bytes=1 << 40):
    return fate.load().fate_attn_paged(h or heads(), s or seqs(), q or rows(), c or cache(), most, scale, out or rows(), None,
                                       None, ws, ws_bytes, None)


def prompt(h=None, s=None, q=None, k=None, v=None, scale=0.1, out=None):
    return fate.load().fate_attn_prompt(h or heads(), s or seqs(), q or rows(), k or rows(), v or rows(), scale, out or rows(),
                                        None, None, None)


BAD_HEADS = [(dict(dtype=2), -1), (dict(dtype=-1), -1), (dict(heads_q=7), -1), (dict(heads_q=0), -1), (dict(heads_kv=0), -1),
             (dict(heads_q=512), -2), (dict(head_dim=0), -1), (dict(head_dim=68), -1), (dict(head_dim=264), -2)]
BAD_SEQS = [(dict(B=-1), -1), (dict(T=-1), -1), (dict(off=None), -1), (dict(T=1 << 30), -2), (dict(B=1 << 25), -2)]
BAD_TABLES = [(dict(kv_len=None), -1), (dict(pages=None), -1), (dict(max_pages=-1), -1), (dict(pages_stride=-1), -1),
              (dict(max_pages=1 << 27), -2)]
BAD_CACHE = [(dict(page_size=0), -1), (dict(page_size=24), -1), (dict(page_size=2048), -2), (dict(k=None), -1), (dict(v=A + 2), -1),
             (dict(page=4), -1), (dict(head=60), -1), (dict(token=8), -1), (dict(n_pages=-1), -1)]
BAD_ROWS = [dict(data=None), dict(data=A + 8), dict(token=12), dict(head=-64), dict(token=-8)]
BAD_OUT = BAD_ROWS + [dict(token=0), dict(head=56)]


@pytest.mark.parametrize("bad,status", BAD_HEADS, ids=str)
def test_heads(bad, status):
    for f in (append, paged, prompt):
        assert f(h=heads(**bad)) == status
    n = C.c_size_t(7)
    assert fate.load().fate_attn_paged_ws_size(heads(**bad), seqs(), cache(), 1, n) == status and n.value == 7


@pytest.mark.parametrize("bad,status", BAD_SEQS, ids=str)
def test_sequences(bad, status):
    for f in (append, paged, prompt):
        assert f(s=seqs(**bad)) == status


@pytest.mark.parametrize("bad,status", BAD_TABLES, ids=str)
def test_tables(bad, status):
    for f in (append, paged):
        assert f(s=seqs(**bad)) == status


@pytest.mark.parametrize("bad,status", BAD_CACHE, ids=str)
def test_cache(bad, status):
    for f in (append, paged):
        assert f(c=cache(**bad)) == status


@pytest.mark.parametrize("bad", BAD_OUT, ids=str)
def test_rows(bad):
    if bad in BAD_ROWS:
        assert append(q=rows(**bad)) == append(k=rows(**bad)) == append(v=rows(**bad)) == -1
        assert paged(q=rows(**bad)) == prompt(q=rows(**bad)) == prompt(k=rows(**bad)) == prompt(v=rows(**bad)) == -1
    assert append(qo=rows(**bad)) == paged(out=rows(**bad)) == prompt(out=rows(**bad)) == -1


def test_others():
    for scale in (0.0, -1.0, float("inf"), float("nan")):
        assert paged(scale=scale) == prompt(scale=scale) == -1
    assert paged(most=-1) == paged(most=7) == -1
    assert paged(ws=None) == paged(ws=A + 4) == -1
    assert paged(ws_bytes=100) == -5
    assert append(rot=66) == append(rot=-2) == append(rot=3) == append(table=None) == append(inter=2) == -1
    assert append(table_rows=-1) == -1
    assert append(q=None) == append(qo=None) == -1
    assert append(q=rows(), qo=rows(token=1024)) == -1  # in place with other strides
    lib = fate.load()
    assert lib.fate_kv_append(None, seqs(), None, rows(), rows(), None, 0, 0, 0, cache(), None, None, None) == -1
    assert lib.fate_kv_append(heads(), None, None, rows(), rows(), None, 0, 0, 0, cache(), None, None, None) == -1
    assert lib.fate_kv_append(heads(), seqs(), None, rows(), rows(), None, 0, 0, 0, None, None, None, None) == -1
    assert lib.fate_attn_paged_ws_size(heads(), seqs(), cache(), 1, None) == -1


def test_nothing_to_do_needs_no_gpu():
    for s in (seqs(B=0), seqs(T=0)):
        assert append(s=s) == prompt(s=s) == 0
        assert paged(s=s, most=0) == 0


def test_workspace_size():
    n = C.c_size_t(0)
    lib = fate.load()
    assert lib.fate_attn_paged_ws_size(heads(), seqs(T=0), cache(), 0, n) == 0 and n.value == 0
    sizes = []
    for most in (1, 4, 6):
        assert lib.fate_attn_paged_ws_size(heads(), seqs(T=64), cache(), most, n) == 0
        sizes.append(n.value)
        assert paged(s=seqs(T=64), most=most, ws_bytes=n.value - 1) == -5
    assert sizes == sorted(sizes) and sizes[0] > 0


def test_mirrors_match_the_header(tmp_path):
    mirrors = [("fate_heads_t", fate.Heads), ("fate_rows_t", fate.Rows), ("fate_kv_cache_t", fate.KvCache),
               ("fate_seqs_t", fate.Seqs)]
    src, want = ["#include <stddef.h>", "#include <stdio.h>", '#include "fate.h"', "int main(void) {"], []
    for c, py in mirrors:
        src.append('printf("%%zu\\n", sizeof(%s));' % c)
        want.append(C.sizeof(py))
        for f, _ in py._fields_:
            src.append('printf("%%zu\\n", offsetof(%s, %s));' % (c, f))
            want.append(getattr(py, f).offset)
    (tmp_path / "a.c").write_text("\n".join(src + ["return 0; }"]))
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    subprocess.run(["gcc", "-std=c11", "-I", os.path.join(root, "include"), str(tmp_path / "a.c"), "-o", str(tmp_path / "a")],
                   check=True)
    out = subprocess.run([str(tmp_path / "a")], check=True, capture_output=True, text=True).stdout
    assert [int(x) for x in out.split()] == want

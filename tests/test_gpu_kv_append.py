"""fate_kv_append against the rotation in 64 bits: what is stored, where, and what is left alone."""

import numpy as np
import pytest
import torch

import attn_oracle as ao
from paper_2605_07238_amd import fate

pytestmark = pytest.mark.gpu


def call(new, kv, hq, hkv, d, dtype, P, rot, interleaved, seed=0, in_place=False, table_rows=None, layout="page"):
    gen = torch.Generator().manual_seed(seed)
    off = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
    T = int(off[-1])
    need = [-(-L // P) for L in kv]
    n_pages = sum(need) + 2
    ids = np.random.default_rng(seed).permutation(n_pages)
    pages, at = np.full((len(new), max(need + [1])), -1, np.int32), 0
    for b, n in enumerate(need):
        pages[b, :n] = ids[at:at + n]
        at += n
    qkv = torch.randn(T, hq + 2 * hkv, d, generator=gen).to(dtype)
    kc, vc = (torch.randn(n_pages, hkv, P, d, generator=gen).to(dtype) for _ in range(2))
    table = fate.rotation_table(table_rows or max(max(kv), 1), rot, device="cpu") if rot else None
    x = qkv.cuda()
    dk, dv = kc.cuda(), vc.cuda()
    if layout == "token":
        dk, dv = (c.transpose(1, 2).contiguous().transpose(1, 2) for c in (dk, dv))
    q = x[:, :hq]
    status = torch.zeros(len(new), dtype=torch.int32, device="cuda")
    got = fate.fate_kv_append(q, x[:, hq:hq + hkv], x[:, hq + hkv:], dk, dv, torch.from_numpy(off).cuda(),
                              torch.tensor(kv, dtype=torch.int32, device="cuda"), torch.from_numpy(pages).cuda(),
                              table.cuda() if rot else None, interleaved=interleaved, q_out=q if in_place else None,
                              status=status)
    assert not status.any()
    if in_place:
        assert got.data_ptr() == x.data_ptr()
        assert torch.equal(x[:, hq:].cpu(), qkv[:, hq:])
    # what must be there
    unit = ao.UNIT[dtype]
    tab = table.double().numpy() if rot else np.zeros((1 << 20, 0))
    want_q, want_k, want_v = qkv[:, :hq].double().numpy().copy(), kc.double().numpy(), vc.double().numpy()
    tol_q, tol_k = np.zeros(want_q.shape), np.zeros(want_k.shape)
    for b in range(len(new)):
        for i in range(new[b]):
            t, pos = off[b] + i, kv[b] - new[b] + i
            if pos < 0:
                want_q[t] = 0
                continue
            row = qkv[t:t + 1].double().numpy()
            y, err = ao.rotate(row, np.array([pos]), tab, interleaved)
            bound = err + unit * (np.abs(y) + err) + ao.TINY
            bound[..., rot:] = 0  # copied as they are
            want_q[t], tol_q[t] = y[0, :hq], bound[0, :hq]
            p, s = pages[b, pos // P], pos % P
            want_k[p, :, s], tol_k[p, :, s] = y[0, hq:hq + hkv], bound[0, hq:hq + hkv]
            want_v[p, :, s] = row[0, hq + hkv:]
    assert (np.abs(got.double().cpu().numpy() - want_q) <= tol_q).all()
    assert (np.abs(dk.double().cpu().numpy() - want_k) <= tol_k).all()
    assert np.array_equal(dv.double().cpu().numpy(), want_v)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16], ids=["bf16", "f16"])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("heads,rot", [((8, 2, 128), 128), ((4, 4, 64), 32), ((20, 4, 80), 80), ((3, 1, 80), 20),
                                       ((2, 2, 256), 64), ((1, 1, 8), 8), ((5, 5, 24), 2), ((4, 2, 64), 0),
                                       ((7, 1, 16), 16), ((2, 1, 104), 16)], ids=str)
def test_append(heads, rot, interleaved, dtype):
    call([1, 0, 40, 3], [1, 5, 300, 129], *heads, dtype, 16, rot, interleaved, seed=rot)


@pytest.mark.parametrize("P", [1, 8, 64, 1024])
def test_page_sizes(P):
    call([5, 1, 130], [70, 4096, 130], 4, 2, 64, torch.bfloat16, P, 64, False, seed=P)


def test_many_tokens_and_sequences():
    rng = np.random.default_rng(3)
    new = rng.integers(0, 20, 150).tolist()
    call(new, [n + int(x) for n, x in zip(new, rng.integers(0, 50, 150))], 2, 1, 64, torch.float16, 16, 64, False)


def test_rows_without_a_place():
    """More new tokens than keys: the first rows stand at negative positions."""
    call([6, 3, 2], [2, 0, 40], 4, 2, 64, torch.bfloat16, 16, 64, False)
    call([6, 3, 2], [2, 0, 40], 4, 2, 64, torch.bfloat16, 16, 20, True)


@pytest.mark.parametrize("rot,interleaved", [(64, False), (64, True), (20, False), (0, False)])
def test_in_place(rot, interleaved):
    call([3, 30], [10, 90], 4, 2, 64, torch.bfloat16, 16, rot, interleaved, in_place=True)


def test_cache_kept_token_by_token():
    call([3, 30], [10, 90], 4, 2, 128, torch.bfloat16, 16, 128, False, layout="token")


def test_without_queries_and_shared_stream():
    k = torch.randn(5, 2, 64).half().cuda()
    c = [torch.zeros(2, 2, 16, 64, dtype=torch.float16, device="cuda") for _ in range(2)]
    i = lambda *x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    assert fate.fate_kv_append(None, k, k, *c, i(0, 5), i(5), i(1).view(1, 1), stream=side) is None
    side.synchronize()
    for x in c:
        assert torch.equal(x[1, :, :5], k.transpose(0, 1)) and not x[0].any() and not x[1, :, 5:].any()


def test_device_errors_store_nothing():
    k = torch.ones(6, 2, 64, dtype=torch.float16, device="cuda")
    i = lambda *x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    table = fate.rotation_table(8, 64)
    for off, kv, pages, bad in ((i(0, 3, 6), i(3, 6), i(0, -1, 2, 1).view(2, 2), None),      # sound
                                (i(0, 3, 6), i(3, 6), i(0, -1, 4, 1).view(2, 2), 1),         # page past the cache
                                (i(0, 3, 6), i(3, 6), i(0, -1, -2, 1).view(2, 2), 1),
                                (i(0, 3, 6), i(33, 6), i(0, 1, 2, 1).view(2, 2), 0),         # more keys than pages hold
                                (i(0, 3, 6), i(3, 10), i(0, -1, 2, 1).view(2, 2), 1),        # position past the table
                                (i(0, 3, 7), i(3, 6), i(0, -1, 2, 1).view(2, 2), 1)):        # rows past T
        c = [torch.zeros(4, 2, 16, 64, dtype=torch.float16, device="cuda") for _ in range(2)]
        status = torch.zeros(2, dtype=torch.int32, device="cuda")
        fate.fate_kv_append(None, k, k, *c, off, kv, pages, table, status=status)
        assert status.tolist() == [fate.FATE_EINVAL if b == bad else 0 for b in range(2)]
        stored = int((c[1] != 0).sum())
        assert stored == 2 * 64 * (6 if bad is None else 4 if int(kv[1]) == 10 else 3)

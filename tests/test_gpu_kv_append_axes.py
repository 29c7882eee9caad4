"""fate_kv_append_axes against the rotation in 64 bits, each pair by its axis's position."""

import numpy as np
import pytest
import torch

import attn_oracle as ao
from paper_2605_07238_amd import fate

pytestmark = pytest.mark.gpu
BF, HF = torch.bfloat16, torch.float16


def ints(x):
    return torch.as_tensor(np.ascontiguousarray(x), dtype=torch.int32).cuda()


def call(new, kv, hq, hkv, d, dtype, P, axis, n_axes, interleaved, seed=0, spoil=(), in_place=False, gap=0):
    """spoil: (token, axis, position) that the table does not have."""
    gen, rng = torch.Generator().manual_seed(seed), np.random.default_rng(seed)
    off = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
    T, half, rows = int(off[-1]), len(axis), 77
    need = [-(-L // P) for L in kv]
    ids, n_pages = rng.permutation(sum(need) + 2), sum(need) + 2
    pages, at = np.full((len(new), max(need + [1])), -1, np.int32), 0
    for b, n in enumerate(need):
        pages[b, :n] = ids[at:at + n]
        at += n
    qkv = torch.randn(T, hq + 2 * hkv, d, generator=gen).to(dtype)
    kc, vc = (torch.randn(n_pages, hkv, P, d, generator=gen).to(dtype) for _ in range(2))
    table = fate.rotation_table(rows, 2 * half, device="cpu")
    turn = rng.integers(0, rows, (n_axes, T)).astype(np.int32)
    bad = set()
    for t, a, value in spoil:
        turn[a, t] = value
        bad.add(int(np.searchsorted(off, t, side="right")) - 1)
    whole = torch.full((n_axes, T + gap), -5, dtype=torch.int32, device="cuda")
    whole[:, :T] = ints(turn)
    x, dk, dv = qkv.cuda(), kc.cuda(), vc.cuda()
    q, status = x[:, :hq], torch.zeros(len(new), dtype=torch.int32, device="cuda")
    got = fate.fate_kv_append_axes(q, x[:, hq:hq + hkv], x[:, hq + hkv:], dk, dv, ints(off), ints(kv), ints(pages), table.cuda(),
                                   whole[:, :T], axis, interleaved=interleaved, q_out=q if in_place else None, status=status)
    assert status.tolist() == [-1 if b in bad else 0 for b in range(len(new))]
    unit, tab = ao.UNIT[dtype], table.double().numpy()
    want_q, want_k, want_v = qkv[:, :hq].double().numpy().copy(), kc.double().numpy(), vc.double().numpy()
    tol_q, tol_k, sure = np.zeros(want_q.shape), np.zeros(want_k.shape), np.ones(T, bool)
    for b in range(len(new)):
        for i in range(new[b]):
            t, pos = off[b] + i, kv[b] - new[b] + i
            if pos < 0:
                want_q[t] = 0
                continue
            if any(not 0 <= p < rows for p in turn[:, t]):
                sure[t] = False  # unspecified; its key and value are not stored
                continue
            of = np.array(axis)
            own = np.concatenate([tab[turn[of, t], np.arange(half)], tab[turn[of, t], half + np.arange(half)]])[None]
            row = qkv[t:t + 1].double().numpy()
            y, err = ao.rotate(row, np.array([0]), own, interleaved)
            bound = err + unit * (np.abs(y) + err) + ao.TINY
            bound[..., 2 * half:] = 0
            want_q[t], tol_q[t] = y[0, :hq], bound[0, :hq]
            p, s = pages[b, pos // P], pos % P
            want_k[p, :, s], tol_k[p, :, s] = y[0, hq:hq + hkv], bound[0, hq:hq + hkv]
            want_v[p, :, s] = row[0, hq + hkv:]
    assert (np.abs(got.double().cpu().numpy() - want_q) <= tol_q)[sure].all()
    assert (np.abs(dk.double().cpu().numpy() - want_k) <= tol_k).all()
    assert np.array_equal(dv.double().cpu().numpy(), want_v)


@pytest.mark.parametrize("dtype", [BF, HF], ids=["bf16", "f16"])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("cyclic", [False, True])
@pytest.mark.parametrize("heads,sections", [((8, 2, 128), (16, 24, 24)), ((4, 4, 64), (3, 5, 8)), ((20, 4, 80), (8, 16, 16)),
                                            ((3, 1, 80), (1, 9)), ((2, 2, 256), (32, 32, 32, 32)), ((1, 1, 8), (1, 1, 1)),
                                            ((5, 5, 24), (1,)), ((7, 1, 16), (2, 2, 2, 2)), ((2, 1, 104), (8, 0, 40)),
                                            ((16, 1, 128), (64,)), ((2, 2, 256), (40, 47, 41))], ids=str)
def test_axes(heads, sections, cyclic, interleaved, dtype):
    axis = fate.rotation_axes(sections, cyclic)
    assert sorted(axis) == [a for a, n in enumerate(sections) for _ in range(n)]
    call([1, 0, 40, 3], [1, 5, 300, 129], *heads, dtype, 16, axis, len(sections), interleaved, seed=len(axis))


@pytest.mark.parametrize("sections", [(16, 24, 24), (24, 20, 20)])
def test_many_tokens(sections):
    """Four tokens a workgroup, and rows read past the last-level cache."""
    call([700, 1, 900], [700, 90, 1000], 8, 2, 128, BF, 16, fate.rotation_axes(sections), 3, False, seed=1, in_place=True, gap=3)


def test_any_order_of_axes_and_unused_ones():
    axis = tuple(int(a) for a in np.random.default_rng(0).integers(0, 3, 32))
    call([5, 9], [5, 40], 4, 2, 64, HF, 8, axis, 4, False)
    call([5, 9], [5, 40], 4, 2, 64, HF, 8, axis, 4, True)


def test_rows_without_a_place_and_positions_out_of_range():
    axis = fate.rotation_axes((16, 24, 24))
    call([6, 3], [4, 3], 4, 2, 128, BF, 16, axis, 3, False)
    for value in (-1, 77, (1 << 31) - 1, -(1 << 31)):
        for a in range(3):
            call([6, 3, 4], [9, 3, 4], 4, 2, 128, BF, 16, axis, 3, False, spoil=[(7, a, value)])
    # rows without a place are not looked at
    call([6], [4], 4, 2, 128, BF, 16, axis, 3, False)


def test_one_axis_is_the_plain_append():
    """The same positions on every axis: the bits that fate_kv_append writes."""
    gen = torch.Generator(device="cuda").manual_seed(0)
    for T in (40, 2000):
        x = torch.randn(T, 12, 128, generator=gen, device="cuda").to(BF)
        P, width = 16, -(-(T + 30) // 16)
        pages, table = ints(np.arange(width)[None]), fate.rotation_table(T + 30, 128)
        caches = [[torch.zeros(width, 2, P, 128, dtype=BF, device="cuda") for _ in range(2)] for _ in range(3)]
        args = [(x[:, :8], x[:, 8:10], x[:, 10:], *c, ints([0, T]), ints([T + 30]), pages, table) for c in caches]
        at = ints(np.stack([np.arange(30, T + 30)] * 3))
        q = [fate.fate_kv_append(*args[0]), fate.fate_kv_append_axes(*args[1], at, fate.rotation_axes((16, 24, 24))),
             fate.fate_kv_append_axes(*args[2], at, fate.rotation_axes((16, 24, 24), cyclic=True))]
        for i in (1, 2):
            assert torch.equal(q[0], q[i]) and torch.equal(caches[0][0], caches[i][0]) and torch.equal(caches[0][1], caches[i][1])


def test_captured_and_on_another_stream():
    axis = fate.rotation_axes((8, 12, 12))
    x = torch.randn(3, 8, 64, device="cuda").to(HF)
    kc, vc = (torch.zeros(4, 2, 4, 64, dtype=HF, device="cuda") for _ in range(2))
    kv, at, table = ints([1, 2, 3]), ints(np.zeros((3, 3))), fate.rotation_table(50, 64)
    pages, off = ints([[0, -1], [1, -1], [2, 3]]), ints([0, 1, 2, 3])
    out = torch.empty(3, 4, 64, dtype=HF, device="cuda")
    go = lambda **m: fate.fate_kv_append_axes(x[:, :4], x[:, 4:6], x[:, 6:], kc, vc, off, kv, pages, table, at, axis, **m)  # noqa: E731
    go(q_out=out)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    other = go(stream=side)
    side.synchronize()
    assert torch.equal(out, other)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        go(q_out=out)
    for step in range(4):
        at += 7
        graph.replay()
        again = go()
        assert torch.equal(out, again)


def test_what_the_binding_refuses():
    axis = fate.rotation_axes((8, 12, 12))
    x = torch.randn(3, 8, 64, device="cuda").to(HF)
    kc, vc = (torch.zeros(4, 2, 4, 64, dtype=HF, device="cuda") for _ in range(2))
    good = dict(q=x[:, :4], k=x[:, 4:6], v=x[:, 6:], k_cache=kc, v_cache=vc, off=ints([0, 3]), kv_len=ints([3]), pages=ints([[0]]),
                table=fate.rotation_table(50, 64), positions=ints(np.zeros((3, 3))), axis=axis)
    assert fate.fate_kv_append_axes(**good).shape == (3, 4, 64)
    wide = ints(np.zeros((3, 6)))
    for name, bad in (("positions", ints(np.zeros((3, 2)))), ("positions", ints(np.zeros(3))), ("positions", wide[:, ::2]),
                      ("positions", good["positions"].long()), ("positions", good["positions"].cpu()), ("axis", axis[1:]),
                      ("axis", (-1,) + axis[1:]), ("axis", (256,) + axis[1:])):
        with pytest.raises(ValueError):
            fate.fate_kv_append_axes(**dict(good, **{name: bad}))
    for name, bad in (("axis", (3,) + axis[1:]), ("positions", ints(np.zeros((5, 3))))):
        with pytest.raises(fate.FateError):
            fate.fate_kv_append_axes(**dict(good, **{name: bad}))
    for name in ("q", "k", "v", "k_cache", "v_cache", "table"):
        with pytest.raises(ValueError, match="gradient"):
            fate.fate_kv_append_axes(**dict(good, **{name: good[name].detach().clone().requires_grad_()}))

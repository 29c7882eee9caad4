"""The calls of a step of answers at their ends: elements past 32 bits, rows and sequences that are not in the call, two calls
at once."""

import numpy as np
import pytest
import torch

from paper_2605_07238_amd import fate
from test_gpu_sample import check, few_values, logits_of, uniform

pytestmark = pytest.mark.gpu
BF, HF, FF = torch.bfloat16, torch.float16, torch.float32


@pytest.fixture(autouse=True, scope="module")
def memory_goes_back():
    yield
    torch.cuda.empty_cache()


def ints(x):
    return torch.as_tensor(np.ascontiguousarray(x), dtype=torch.int32).cuda()


def step(cache, pages, new, kv, qkv, lead=0, trail=0, **more):
    """Append by two axes, then windows of 50 keys behind a prefix of 5; results in the call's rows, 3 elsewhere."""
    T = sum(new)
    off = ints(np.concatenate([[0], np.cumsum(new)]) + lead)
    rows = torch.full((lead + T + trail, *qkv.shape[1:]), float("nan"), dtype=qkv.dtype, device="cuda")
    rows[lead:lead + T] = qkv
    pos = np.concatenate([L - n + np.arange(n) for n, L in zip(new, kv)])
    places = torch.full((2, lead + T + trail), -1, dtype=torch.int32, device="cuda")
    places[:, lead:lead + T] = ints([pos, pos // 3])
    start = torch.full((lead + T + trail,), 1 << 30, dtype=torch.int32, device="cuda")
    start[lead:lead + T] = ints(pos - 49)
    q, out = (torch.full((lead + T + trail, 4, 64), 3.0, dtype=qkv.dtype, device="cuda") for _ in range(2))
    status = torch.zeros(len(new), dtype=torch.int32, device="cuda")
    fate.fate_kv_append_axes(rows[:, :4], rows[:, 4:6], rows[:, 6:], *cache, off, ints(kv), pages, fate.rotation_table(600, 64), places,
                             fate.rotation_axes((20, 12)), q_out=q, status=status)
    fate.fate_attn_paged_shaped(q, *cache, off, ints(kv), pages, cap=9.0, slopes=torch.full((4,), 0.01, device="cuda"),
                                prefix=ints([5] * len(new)), start=start, out=out, status=status, **more)
    assert not status.any()
    for x in (q, out):
        assert (x[:lead] == 3).all() and (x[lead + T:] == 3).all()
    return q[lead:lead + T], out[lead:lead + T]


@pytest.mark.parametrize("new", [[1, 1, 1], [3, 1, 7], [80, 2, 130]], ids=str)
def test_pages_past_32_bits_and_rows_outside(new):
    """The same keys in pages at the two ends of a cache of 2^31 elements and more, and the same rows among others."""
    kv, n_pages = [400, 33, 250], (1 << 31) // (2 * 16 * 64) + 60
    caches = [torch.zeros(n_pages, 2, 16, 64, dtype=HF, device="cuda") for _ in range(2)]
    assert caches[0].numel() > 1 << 31
    gen = torch.Generator(device="cuda").manual_seed(sum(new))
    qkv = torch.randn(sum(new), 8, 64, generator=gen, device="cuda").half()
    keys = torch.randn(2, 60, 2, 16, 64, generator=gen, device="cuda").half()
    tables, at = np.full((3, 30), -1), 0
    for b, L in enumerate(kv):
        n = -(-L // 16)
        tables[b, :n] = np.arange(at, at + n)
        at += n
    got = []
    for base, lead, trail in ((0, 0, 0), (n_pages - 60, 0, 0), (n_pages - 60, 11, 5)):
        for c, x in zip(caches, keys):
            c[base:base + 60] = x
        pages = ints(np.where(tables < 0, -1, tables + base))
        got.append(step(caches, pages, new, kv, qkv, lead, trail, max_new=max(new)))  # (the cut of the work follows from it)
        got[-1] += (caches[0][base:base + 60].clone(), caches[1][base:base + 60].clone())
    for other in got[1:]:
        for x, y in zip(got[0], other):
            assert torch.equal(x, y)


@pytest.mark.parametrize("dtype", [BF, FF], ids=["bf16", "f32"])
def test_rows_of_logits_past_32_bits(dtype):
    V, stride = 20011, (1 << 30) + 3
    x = logits_of(3, V, dtype, 7)
    wide = torch.empty(2 * stride + V, dtype=dtype, device="cuda").as_strided((3, V), (stride, 1))

    def far(t):
        wide.copy_(t)
        return wide

    for filters in (dict(top_p=0.9), dict(top_k=30), dict(top_k=700, top_p=0.99), dict()):
        check(x, uniform(3, 9), far, **filters)


def test_two_calls_at_once_and_a_graph_whose_rows_change_their_way():
    """Calls on two streams with workspaces of their own; a captured call whose settings and logits move rows between the
    ways a row can be sampled."""
    R, V = 20, 131072
    x = few_values("plain", R, V, BF, 0).cuda()
    u = torch.rand(R, generator=torch.Generator().manual_seed(1)).cuda()
    p, k = torch.full((R,), 0.9, device="cuda"), ints([0] * R)
    want = fate.fate_sample(x, u, top_p=p, top_k=k)[0]
    torch.cuda.synchronize()
    sides = [torch.cuda.Stream() for _ in range(2)]
    got = [[] for _ in sides]
    for _ in range(6):
        for s, kept in zip(sides, got):
            kept.append(fate.fate_sample(x, u, top_p=p, top_k=k, stream=s)[0])
    torch.cuda.synchronize()
    assert all(torch.equal(t, want) for kept in got for t in kept)
    out = torch.empty(R, dtype=torch.int32, device="cuda")
    ws = torch.empty(fate.fate_sample_ws_size(x), dtype=torch.uint8, device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        fate.fate_sample(x, u, top_p=p, top_k=k, out=out, ws=ws)
    for kind in ("plain", "infinite", "crowded", "wide", "holes", "plain"):
        rng = np.random.default_rng(len(kind))
        x.copy_(few_values(kind, R, V, BF, 3))
        k.copy_(ints(rng.choice([0, 1, 40, 300, 5000], R)))
        p.copy_(torch.tensor(rng.choice([1.0, 0.9, 0.3], R), dtype=torch.float32))
        graph.replay()
        # each row by itself, its settings numbers: launches of another form
        for r in range(R):
            own = fate.fate_sample(x[r:r + 1], u[r:r + 1], top_p=float(p[r]), top_k=int(k[r]))[0]
            assert own[0] == out[r], (kind, r)

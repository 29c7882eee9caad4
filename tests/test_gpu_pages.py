"""fate_kv_reserve and fate_kv_trim against their definitions, sequence by sequence: whole numbers, equal."""

import numpy as np
import pytest
import torch

import serve_oracle as so
from paper_2605_07238_amd import fate

pytestmark = pytest.mark.gpu


def ints(x, dtype=torch.int32):
    return torch.as_tensor(np.ascontiguousarray(x), dtype=dtype).cuda()


def tables(kv, P, width, rng, more):
    """Pages of sequences of these lengths in no order, -1 past them, and the other pages."""
    need = [-(-max(n, 0) // P) for n in kv]
    order = rng.permutation(sum(need) + more)
    pages, at = np.full((len(kv), width), -1, np.int32), 0
    for b, n in enumerate(need):
        n = min(n, width)
        pages[b, :n] = order[at:at + n]
        at += n
    return pages, order[at:]


def reserve(new, kv, pages, free, n_free, P, T, stride=0, in_place=False):
    """The call, against the oracle; its results as the oracle has them."""
    B, width = pages.shape
    whole = torch.full((B, width + stride), -7, dtype=torch.int32, device="cuda")
    dp = whole[:, :width]
    dp.copy_(ints(pages))
    dn, dk, df, dc = ints(new), ints(kv), ints(free), ints([n_free])
    status = torch.zeros(B, dtype=torch.int32, device="cuda")
    out = None
    if in_place:
        out = fate.Reserved(ints(np.full(B + 1, -9)), dk, dc, ints(np.full(B + 1, -9)), ints(np.full(T, -9), torch.int64),
                            ints(np.full(T, -9)))
    got = fate.fate_kv_reserve(dn, dk, dp, df, dc, P, T, out=out, status=status)
    assert not in_place or got is out
    want = so.reserve(list(new), list(kv), pages, list(free), n_free, P, T)
    for name, g, w in zip(got._fields + ("pages", "status"), tuple(got) + (dp, status), want):
        assert np.array_equal(g.cpu().numpy(), w), name
    assert torch.equal(df, ints(free)) and (whole[:, width:] == -7).all()
    if not in_place:
        assert torch.equal(dk, ints(kv)) and dc.item() == n_free
    return want


def random_case(B, P, most_new, most_kv, seed, spare=1.0, room=1.0):
    rng = np.random.default_rng(seed)
    new, kv = rng.integers(0, most_new + 1, B), rng.integers(0, most_kv + 1, B)
    width = int(-(-(kv + new).max() // P)) + 1
    need = int((-(-(kv + new) // P) - -(-kv // P)).sum())
    pages, free = tables(kv, P, width, rng, int(need * spare))
    n_free = len(free)
    free = np.concatenate([free, np.full(int((-(-kv // P)).sum()), -1)])
    return new, kv, pages, free, n_free, P, int(new.sum() * room)


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("B,P,most_new,most_kv", [(1, 16, 1, 100), (1, 1, 5, 5), (64, 16, 1, 4096), (3, 1024, 2000, 5000),
                                                  (63, 8, 40, 200), (65, 2, 70, 30), (1023, 16, 3, 50), (1025, 16, 9, 50),
                                                  (4096, 4, 1, 9), (4097, 4, 2, 9), (9000, 16, 0, 40), (17, 16, 4000, 100),
                                                  (2500, 32, 30, 64)], ids=str)
def test_reserve(B, P, most_new, most_kv, in_place):
    reserve(*random_case(B, P, most_new, most_kv, B + P), in_place=in_place)


@pytest.mark.parametrize("spare,room", [(0.0, 1.0), (0.5, 1.0), (0.97, 1.0), (1.0, 0.0), (1.0, 0.4), (0.6, 0.7), (2.0, 1.5)])
@pytest.mark.parametrize("B", [7, 300, 2000])
def test_too_few_pages_or_rows(B, spare, room):
    want = reserve(*random_case(B, 16, 40, 100, B, spare, room), stride=5)
    assert (want[-1] != 0).any() == (spare < 1 or room < 1)


def test_rows_on_both_sides_of_one_launch():
    for T in (4095, 4096, 4097, 5121):
        rng = np.random.default_rng(T)
        pages, free = tables([0, 3], 16, 400, rng, 400)
        reserve([T - 7, 7], [0, 3], pages, np.concatenate([free, [0]]), len(free), 16, T)


def test_sequences_in_error():
    rng = np.random.default_rng(5)
    new, kv = [3, -1, 2, 50, 4, 1, 1 << 30, 2, 0], [5, 6, -4, 30, 1, 64, 5, (1 << 31) - 2, 1 << 30]
    pages, free = tables([5, 6, 0, 30, 1, 64, 5, 0, 0], 16, 4, rng, 20)
    pages[4, 0] = 999  # its own page is out of range: its rows there have no slot
    status = reserve(new, kv, pages, free, 20, 16, 40)[-1]
    assert status.tolist() == [0, -1, -1, -1, -1, -1, -1, -1, -1]


@pytest.mark.parametrize("n_free", [-1, -(1 << 31), 21, (1 << 31) - 1])
def test_counts_that_no_stack_has(n_free):
    rng = np.random.default_rng(6)
    pages, free = tables([15, 16], 16, 4, rng, 17)  # twenty pages, seventeen free
    free = np.concatenate([free, [-1, -1, -1]])
    assert reserve([1, 1], [15, 16], pages, free, n_free, 16, 2)[-1].tolist() == [0, -5]


def test_a_stack_that_holds_no_pages():
    pages = np.full((2, 3), -1, np.int32)
    assert reserve([4, 20], [0, 0], pages, [77, -1, 2], 3, 16, 24)[-1].tolist() == [0, -1]


def test_no_sequences_and_no_rows():
    empty = torch.empty(0, dtype=torch.int32, device="cuda")
    got = fate.fate_kv_reserve(empty, empty, empty.view(0, 4), ints([1, 0]), ints([2]), 16, 5)
    assert got.off.tolist() == got.taken.tolist() == [0] and got.n_free.tolist() == [2]
    assert got.slots.tolist() == got.positions.tolist() == [-1] * 5
    assert fate.fate_kv_trim(empty, empty, empty.view(0, 4), ints([1, 0]), ints([2]), 16).n_free.tolist() == [2]
    reserve([0, 0], [3, 0], np.array([[1, -1], [-1, -1]], np.int32), [0, -1], 1, 16, 0)
    reserve([1 << 30, 0], [3, 0], np.array([[1, -1], [-1, -1]], np.int32), [0, -1], 1, 16, 0)


def test_more_tokens_than_32_bits():
    B = 9000  # sums of what is asked pass 2^32; one page of many is free
    pages = np.full((B, 1 << 10), -1, np.int32)
    new = np.full(B, 1 << 20)
    new[0] = 1000
    status = reserve(new, np.zeros(B, np.int64), pages, np.arange(4), 4, 1024, 1 << 20)[-1]
    assert status[0] == 0 and (status[1:] == -5).all()


def trim(keep, kv, pages, free, n_free, P, in_place=False):
    B = len(keep)
    dk, dp, df, dc = ints(kv), ints(pages), ints(free), ints([n_free])
    status = torch.zeros(B, dtype=torch.int32, device="cuda")
    out = fate.Trimmed(dk, dc, ints(np.full(B + 1, -9))) if in_place else None
    got = fate.fate_kv_trim(ints(keep), dk, dp, df, dc, P, out=out, status=status)
    want = so.trim(list(keep), list(kv), pages, free, n_free, P)
    for name, g, w in zip(("kv_len", "n_free", "given", "free", "status"), tuple(got) + (df, status), want):
        assert np.array_equal(g.cpu().numpy(), w), name
    assert torch.equal(dp, ints(pages))
    return want


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("B,P,most", [(1, 16, 100), (64, 16, 4096), (65, 1, 300), (255, 8, 1500), (256, 4, 1100), (257, 4, 1100), (511, 8, 100), (513, 8, 100), (1025, 16, 90),
                                      (5000, 4, 60), (3, 16, 100000)], ids=str)
def test_trim(B, P, most, in_place):
    rng = np.random.default_rng(B)
    kv = rng.integers(0, most + 1, B)
    keep = np.where(rng.random(B) < 0.3, 0, rng.integers(0, most + 1, B))
    pages, free = tables(kv, P, int(-(-kv.max() // P)) + 2, rng, 9)
    trim(keep, kv, pages, np.concatenate([free, np.full(int((-(-kv // P)).sum()), -1)]), 9, P, in_place)


@pytest.mark.parametrize("n_free", [-3, 0, 3, 6, 9, 40])
@pytest.mark.parametrize("many", [0, 600])
def test_trim_in_error(n_free, many):
    """Lengths and pages out of range, and more pages than the stack has room for."""
    keep, kv = [0, -1, 3, 0, 0, 200, 0] + [0] * many, [20, 20, -1, 200, 16, 64, 33] + [5] * many
    pages = np.arange(7 * 4).reshape(7, 4).astype(np.int32) % 12
    pages[4, 0] = 12
    pages = np.concatenate([pages, np.full((many, 4), 3, np.int32)])
    assert trim(keep, kv, pages, np.arange(100, 112), n_free, 16)[-1][:5].tolist()[1:] == [-1, -1, -1, -1]


@pytest.mark.parametrize("B", [5, 700])
def test_a_stack_over_many_steps(B):
    """Requests come, grow and end, with everything updated in place: no page is ever in two places."""
    P, n_pages, width = 16, 40 * B // 10, 40
    rng = np.random.default_rng(B)
    pages, kv = torch.full((B, width), -1, dtype=torch.int32, device="cuda"), ints(np.zeros(B))
    free, n_free = torch.arange(n_pages, dtype=torch.int32, device="cuda"), ints([n_pages])
    status = torch.zeros(B, dtype=torch.int32, device="cuda")
    i32 = lambda n: torch.empty(n, dtype=torch.int32, device="cuda")  # noqa: E731
    room, cut = fate.Reserved(i32(B + 1), kv, n_free, i32(B + 1), None, None), fate.Trimmed(kv, n_free, i32(B + 1))
    refused = 0
    for step in range(30):
        fate.fate_kv_reserve(ints(rng.integers(0, 60, B)), kv, pages, free, n_free, P, 60 * B, out=room, status=status)
        refused += int((status == -5).sum())
        assert ((status == 0) | (status == -5)).all()
        status.zero_()
        if step % 3 == 2:
            fate.fate_kv_trim(ints(np.where(rng.random(B) < 0.4, 0, rng.integers(0, 600, B))), kv, pages, free, n_free, P, out=cut,
                              status=status)
            assert not status.any()
        have = (kv.cpu().numpy() + P - 1) // P
        held = np.concatenate([pages[b, :have[b]].cpu().numpy() for b in range(B)])
        everything = np.concatenate([held, free[:n_free.item()].cpu().numpy()])
        assert np.array_equal(np.sort(everything), np.arange(n_pages))
    assert refused > 0


def test_captured_and_replayed():
    """A decoding step's tables in a graph: lengths and stack go on in place from replay to replay."""
    P, B = 4, 6
    pages = torch.full((B, 50), -1, dtype=torch.int32, device="cuda")
    kv, free, n_free = ints(np.zeros(B)), torch.arange(B * 50, dtype=torch.int32, device="cuda"), ints([B * 50])
    new, i32 = ints(np.ones(B)), lambda n: torch.empty(n, dtype=torch.int32, device="cuda")  # noqa: E731
    out = fate.Reserved(i32(B + 1), kv, n_free, i32(B + 1), i32(B).long(), i32(B))
    fate.fate_kv_reserve(new, kv, pages, free, n_free, P, B, out=out)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        fate.fate_kv_reserve(new, kv, pages, free, n_free, P, B, out=out)
    for step in range(1, 40):
        before = pages.cpu().numpy(), int(n_free)
        graph.replay()
        torch.cuda.synchronize()
        want = so.reserve([1] * B, [step] * B, before[0], list(range(B * 50)), before[1], P, B)
        for g, w in zip(tuple(out) + (pages,), want):
            assert np.array_equal(g.cpu().numpy(), w)


def test_what_the_binding_refuses():
    good = dict(new=ints([1, 1]), kv_len=ints([3, 0]), pages=ints(np.full((2, 4), 0)), free=ints([1, 2, 3]), n_free=ints([3]),
                page_size=16, T=2)
    assert fate.fate_kv_reserve(**good).off.tolist() == [0, 1, 2]
    for name, bad in (("new", ints([1])), ("new", ints([1, 1], torch.int64)), ("kv_len", ints([3, 0, 0])), ("pages", ints([0, 0])),
                      ("pages", ints(np.zeros((4, 2))).t()), ("free", ints([[1, 2]])), ("free", ints(np.arange(6))[::2]),
                      ("n_free", ints([3, 3])), ("n_free", torch.ones(1, dtype=torch.int32)), ("T", -1)):
        with pytest.raises(ValueError):
            fate.fate_kv_reserve(**dict(good, **{name: bad}))
    for size in (0, 24, 2048):
        with pytest.raises(fate.FateError):
            fate.fate_kv_reserve(**dict(good, page_size=size))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = fate.fate_kv_reserve(**good, stream=side)
    side.synchronize()
    assert got.kv_len.tolist() == [4, 1]


def test_numbers_past_their_types_are_refused():
    """Not taken by their low bits."""
    good = dict(kv_len=ints([3, 0]), pages=ints(np.full((2, 4), 0)), free=ints([1, 2, 3]), n_free=ints([3]), page_size=16)
    for size in ((1 << 32) + 16, 16 - (1 << 32), 1 << 31, 1 << 70):
        with pytest.raises(ValueError):
            fate.fate_kv_reserve(ints([1, 1]), T=2, **dict(good, page_size=size))
        with pytest.raises(ValueError):
            fate.fate_kv_trim(ints([1, 0]), **dict(good, page_size=size))
    out = fate.Reserved(ints([0] * 3), ints([0] * 2), ints([0]), ints([0] * 3), None, None)
    for T in ((1 << 64) + 2, 2 - (1 << 64), -1):
        with pytest.raises(ValueError):
            fate.fate_kv_reserve(ints([1, 1]), T=T, out=out, **good)
    assert fate.fate_kv_reserve(ints([1, 1]), T=2, out=out, **good).off.tolist() == [0, 1, 2]

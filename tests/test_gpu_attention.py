"""fate_attn_paged and fate_attn_prompt against attention in 64 bits.

Bounds are derived in attn_oracle.py from the kernels' arithmetic: float32
sums and statistics, weights and results rounded to the operands' type."""

import math

import numpy as np
import pytest
import torch

import attn_oracle as ao
from paper_2605_07238_amd import fate

pytestmark = pytest.mark.gpu
BF, HF = torch.bfloat16, torch.float16


def compare(got, lse, want):
    out, ref_lse, tol, tol_lse = want
    g = got.double().cpu().numpy()
    assert np.isfinite(g).all()
    off = np.abs(g - out) - tol
    assert (off <= 0).all(), "worst excess %.3g at %s" % (off.max(), np.unravel_index(off.argmax(), off.shape))
    if lse is not None:
        s = lse.double().cpu().numpy()
        empty = np.isneginf(ref_lse)
        assert np.array_equal(np.isneginf(s), empty)
        assert (np.abs(s - ref_lse)[~empty] <= tol_lse[~empty]).all()


def make_paged(new, kv, hq, hkv, d, dtype, P, seed=0, scale_q=1.0, spare=3):
    """CPU tensors and lists of a paged call: kv[b] keys with the new[b] tokens among them, pages in no order, -1 past the
    end, a NaN in every slot that no sequence owns."""
    gen = torch.Generator().manual_seed(seed)
    rng = np.random.default_rng(seed)
    need = [-(-L // P) for L in kv]
    n_pages = sum(need) + spare
    ids = rng.permutation(n_pages)
    width = max(need + [1]) + 1
    pages, at = np.full((len(new), width), -1, np.int32), 0
    kc = torch.full((n_pages, hkv, P, d), math.nan, dtype=dtype)
    vc = torch.full((n_pages, hkv, P, d), math.nan, dtype=dtype)
    for b, L in enumerate(kv):
        pages[b, :need[b]] = ids[at:at + need[b]]
        at += need[b]
        for j in range(need[b]):
            n = min(P, L - j * P)
            for c in (kc, vc):
                c[int(pages[b, j]), :, :n] = torch.randn(hkv, n, d, generator=gen).to(dtype)
    off = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
    q = (torch.randn(int(off[-1]), hq, d, generator=gen) * scale_q).to(dtype)
    return q, kc, vc, off, np.array(kv, np.int32), pages


def run_paged(q, kc, vc, off, kv, pages, **more):
    dev = [t.cuda() for t in (q, kc, vc, torch.from_numpy(off), torch.from_numpy(kv), torch.from_numpy(pages))]
    return fate.fate_attn_paged(*dev, lse=True, **more)


# new tokens and keys per sequence: one token over short and long axes, tile and page edges, empty sequences, more new
# tokens than keys (rows that see nothing), nothing cached, no keys at all
LENGTHS = [
    ([1], [1]),
    ([1, 1, 1, 1], [64, 65, 127, 700]),
    ([1, 0, 3, 2, 0], [5, 0, 2, 0, 7]),
    ([5, 5, 4], [300, 5, 33]),
    ([17, 31, 1], [17, 600, 257]),
    ([130, 1, 64, 63], [130, 1, 500, 191]),
    ([200], [1000]),
]
HEADS = [(8, 8, 64), (8, 2, 128), (14, 2, 128), (5, 1, 256), (4, 2, 80), (3, 3, 8), (16, 1, 128)]


@pytest.mark.parametrize("heads", HEADS, ids=str)
@pytest.mark.parametrize("lengths", range(len(LENGTHS)))
def test_paged(heads, lengths):
    new, kv = LENGTHS[lengths]
    P = [16, 1, 8, 64, 16, 32, 256][(lengths + HEADS.index(heads)) % 7]
    dtype = BF if (lengths + heads[2]) % 2 else HF
    args = make_paged(new, kv, *heads, dtype, P, seed=lengths)
    scale = 1 / math.sqrt(heads[2])
    want = ao.paged(*args[:3], args[3].tolist(), args[4].tolist(), args[5].tolist(), scale)
    status = torch.zeros(len(new), dtype=torch.int32, device="cuda")
    out, lse = run_paged(*args, max_new=max(new), status=status)
    compare(out, lse, want)
    # no bound on the new tokens: the kernels for chunks
    out, lse = run_paged(*args, status=status)
    compare(out, lse, want)
    assert not status.any()


@pytest.mark.parametrize("dtype", [BF, HF], ids=["bf16", "f16"])
@pytest.mark.parametrize("new", [1, 4, 9, 40])
def test_paged_split_axis(dtype, new):
    """Few rows over long axes of different lengths: the key axis is split and joined."""
    args = make_paged([new, new, new], [4099, 129, 9001], 8, 2, 128, dtype, 16, seed=new)
    want = ao.paged(*args[:3], args[3].tolist(), args[4].tolist(), args[5].tolist(), 0.1)
    out, lse = run_paged(*args, max_new=new, scale=0.1)
    compare(out, lse, want)
    again, lse2 = run_paged(*args, max_new=new, scale=0.1)
    assert torch.equal(out, again) and torch.equal(lse, lse2)


@pytest.mark.parametrize("scale_q", [0.0, 30.0])
def test_paged_flat_and_peaked(scale_q):
    args = make_paged([3, 70], [1500, 900], 4, 2, 64, HF, 32, seed=3, scale_q=scale_q)
    want = ao.paged(*args[:3], args[3].tolist(), args[4].tolist(), args[5].tolist(), 0.125)
    for most in (70, None):
        compare(*run_paged(*args, max_new=most, scale=0.125), want)


@pytest.mark.parametrize("max_new", [4, 300])
@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
def test_paged_unseen_keys_do_not_reach_a_row(bad, max_new):
    """Infinities and NaN at later positions: rows before them are as without them; rows at them are not finite."""
    n = 4 if max_new == 4 else 300
    args = make_paged([n], [n + 100], 4, 2, 128, BF, 16, seed=9)
    q, kc, vc, off, kv, pages = args
    want = ao.paged(*args[:3], args[3].tolist(), args[4].tolist(), args[5].tolist(), 1 / math.sqrt(128))
    at = 100 + n // 2  # position of the first bad key, seen by rows n // 2 and later
    for c in (kc, vc):
        for j in (at, at + 1):
            c[int(pages[0, j // 16]), :, j % 16] = bad
    out, lse2 = run_paged(*args, max_new=max_new)
    compare(out[:n // 2], lse2[:n // 2], [x[:n // 2] for x in want])
    assert not torch.isfinite(out[n // 2:]).any()


@pytest.mark.parametrize("heads", [(8, 8, 64), (8, 2, 128), (5, 1, 256), (4, 2, 80), (7, 1, 16)], ids=str)
@pytest.mark.parametrize("dtype", [BF, HF], ids=["bf16", "f16"])
def test_prompt(heads, dtype):
    hq, hkv, d = heads
    lens = [1, 64, 0, 65, 31, 127, 333, 2]
    off = np.concatenate([[0], np.cumsum(lens)]).astype(np.int32)
    gen = torch.Generator().manual_seed(d)
    qkv = torch.randn(int(off[-1]), hq + 2 * hkv, d, generator=gen).to(dtype)
    q, k, v = qkv[:, :hq], qkv[:, hq:hq + hkv], qkv[:, hq + hkv:]
    want = ao.prompt(q, k, v, off.tolist(), 1 / math.sqrt(d))
    x = qkv.cuda()
    status = torch.zeros(len(lens), dtype=torch.int32, device="cuda")
    out, lse = fate.fate_attn_prompt(x[:, :hq], x[:, hq:hq + hkv], x[:, hq + hkv:], torch.from_numpy(off).cuda(), lse=True,
                                     status=status)
    compare(out, lse, want)
    assert not status.any()


@pytest.mark.parametrize("bad", [math.nan, math.inf])
def test_prompt_later_tokens_do_not_reach_earlier_rows(bad):
    gen = torch.Generator().manual_seed(1)
    q, k, v = (torch.randn(200, 2, 64, generator=gen).half() for _ in range(3))
    want = ao.prompt(q, k, v, [0, 77, 200], 0.125)
    q, k, v = q.cuda(), k.cuda(), v.cuda()
    off = torch.tensor([0, 77, 200], dtype=torch.int32, device="cuda")
    k[60:77], v[60:77] = bad, bad
    k[190], v[190] = bad, bad
    out, lse = fate.fate_attn_prompt(q, k, v, off, lse=True)
    for rows in (slice(0, 60), slice(77, 190)):
        compare(out[rows], lse[rows], [x[rows] for x in want])
    assert not torch.isfinite(out[60:77]).any() and not torch.isfinite(out[190:]).any()


def test_prompt_agrees_with_the_cache():
    """A prompt attended whole, and appended and attended in two chunks over the cache: within the bounds of both."""
    gen = torch.Generator().manual_seed(2)
    n, cut, hq, hkv, d, P = 300, 170, 8, 2, 128, 16
    q, k, v = (torch.randn(n, h, d, generator=gen).to(BF) for h in (hq, hkv, hkv))
    want = ao.prompt(q, k, v, [0, n], 0.088)
    q, k, v = q.cuda(), k.cuda(), v.cuda()
    kc = torch.empty(32, hkv, P, d, dtype=BF, device="cuda")
    vc = torch.empty_like(kc)
    pages = torch.randperm(32, generator=gen)[:20].view(1, -1).int().cuda()
    parts = []
    for lo, hi in ((0, cut), (cut, n)):
        off, kv = (torch.tensor(x, dtype=torch.int32, device="cuda") for x in ([0, hi - lo], [hi]))
        rows = fate.fate_kv_append(q[lo:hi], k[lo:hi], v[lo:hi], kc, vc, off, kv, pages)
        parts.append(fate.fate_attn_paged(rows, kc, vc, off, kv, pages, scale=0.088, lse=True))
    compare(torch.cat([p[0] for p in parts]), torch.cat([p[1] for p in parts]), want)
    out, lse = fate.fate_attn_prompt(q, k, v, torch.tensor([0, n], dtype=torch.int32, device="cuda"), scale=0.088, lse=True)
    compare(out, lse, want)


def test_strides():
    """A cache kept token by token, queries and results kept head by head, keys that all tokens share."""
    args = make_paged([3, 90], [200, 333], 4, 2, 64, BF, 16, seed=5)
    q, kc, vc, off, kv, pages = args
    want = ao.paged(q, kc, vc, off.tolist(), kv.tolist(), pages.tolist(), 0.125)
    wide = torch.full((93, 4, 200), 7.0, dtype=BF, device="cuda")
    for most in (90, None, 3):
        tk, tv = (c.transpose(1, 2).contiguous().cuda().transpose(1, 2) for c in (kc, vc))
        qh = q.transpose(0, 1).contiguous().cuda().transpose(0, 1)
        out = torch.empty(4, 93, 64, dtype=BF, device="cuda").transpose(0, 1)
        tables = torch.full((2, 50), -1, dtype=torch.int32, device="cuda")
        tables[:, :pages.shape[1]] = torch.from_numpy(pages).cuda()
        got, lse = fate.fate_attn_paged(qh, tk, tv, torch.from_numpy(off).cuda(), torch.from_numpy(kv).cuda(),
                                        tables[:, :pages.shape[1]], max_new=most, out=out, lse=True)
        assert got.data_ptr() == out.data_ptr()
        compare(out, lse, want)
        fate.fate_attn_paged(qh, tk, tv, torch.from_numpy(off).cuda(), torch.from_numpy(kv).cuda(), tables, max_new=most,
                             out=wide[:, :, 8:72])
        assert torch.equal(wide[:, :, 8:72], out)
        assert (wide[:, :, :8] == 7).all() and (wide[:, :, 72:] == 7).all()
    gen = torch.Generator().manual_seed(0)
    q = torch.randn(50, 4, 64, generator=gen).to(BF)
    k = torch.randn(1, 2, 64, generator=gen).to(BF).expand(50, 2, 64)
    v = torch.randn(50, 1, 64, generator=gen).to(BF).expand(50, 2, 64)
    off = torch.tensor([0, 50], dtype=torch.int32, device="cuda")
    out, lse = fate.fate_attn_prompt(q.cuda(), k[:1].cuda().expand(50, 2, 64), v[:, :1].cuda().expand(50, 2, 64), off, lse=True)
    compare(out, lse, ao.prompt(q, k, v, [0, 50], 0.125))


def test_rows_outside_sequences_are_left_alone():
    args = make_paged([2, 66], [40, 300], 4, 2, 64, BF, 16, seed=6)
    q, kc, vc, off, kv, pages = args
    want = ao.paged(q, kc, vc, off.tolist(), kv.tolist(), pages.tolist(), 0.125)
    padded = torch.full((5 + 68 + 9, 4, 64), math.nan, dtype=BF)
    padded[5:73] = q
    for most in (66, None, 2):
        out = torch.full((82, 4, 64), 3.0, dtype=BF, device="cuda")
        got, lse = run_paged(padded, kc, vc, off + 5, kv, pages, max_new=most, out=out)
        compare(out[5:73], lse[5:73], want)
        assert (out[:5] == 3).all() and (out[73:] == 3).all()


def test_offsets_past_32_bits():
    """Pages whose elements lie past 2^31 and bytes past 2^32, in a cache of 9 GB."""
    hkv, P, d = 2, 64, 128
    n_pages = 9 * (1 << 30) // 2 // (2 * hkv * P * d)
    kc = torch.zeros(n_pages, hkv, P, d, dtype=BF, device="cuda")
    vc = torch.zeros_like(kc)
    assert kc.numel() > 2 ** 31
    used = [n_pages - 1, 3, n_pages - 7, n_pages // 2 + 1]
    gen = torch.Generator().manual_seed(8)
    pages = torch.tensor([used], dtype=torch.int32, device="cuda")
    L = 4 * P - 5
    for n in (1, 100):
        q, k, v = (torch.randn(m, h, d, generator=gen).to(BF) for m, h in ((n, 4), (L, hkv), (L, hkv)))
        one = lambda *x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
        fate.fate_kv_append(None, k.cuda(), v.cuda(), kc, vc, one(0, L), one(L), pages)
        small_k = torch.stack([kc[p] for p in used]).cpu()
        small_v = torch.stack([vc[p] for p in used]).cpu()
        assert torch.equal(small_k.transpose(1, 2).reshape(-1, hkv, d)[:L], k)
        out, lse = fate.fate_attn_paged(q.cuda(), kc, vc, one(0, n), one(L), pages, max_new=n, lse=True)
        compare(out, lse, ao.paged(q, small_k, small_v, [0, n], [L], [[0, 1, 2, 3]], 1 / math.sqrt(d)))


def test_device_errors_are_reported_and_contained():
    """Page numbers, lengths and offsets out of range: FATE_EINVAL for their sequence, the others' results as ever."""
    args = make_paged([2, 70, 1, 3], [200, 100, 300, 64], 4, 2, 64, BF, 16, seed=4)
    q, kc, vc, off, kv, pages = args
    for most in (3, 70):
        good, _ = run_paged(*args, max_new=most)
        for what in ("page", "page-", "kv", "kv-"):
            kv2, pages2 = kv.copy(), pages.copy()
            if what == "page":
                pages2[2, 1] = kc.shape[0]
            elif what == "page-":
                pages2[2, 18] = -1
            elif what == "kv":
                kv2[2] = 16 * pages.shape[1] + 1
            else:
                kv2[2] = -5
            status = torch.zeros(4, dtype=torch.int32, device="cuda")
            out, _ = run_paged(q, kc, vc, off, kv2, pages2, max_new=most, status=status)
            assert status.tolist() == [0, 0, fate.FATE_EINVAL, 0], what
            keep = [0, 1, *range(2, 72), *range(73, 76)]
            assert torch.equal(out[keep], good[keep]), what
    off2 = off.copy()
    off2[4] = 90  # past the rows
    status = torch.zeros(4, dtype=torch.int32, device="cuda")
    out, _ = run_paged(q, kc, vc, off2, kv, pages, max_new=70, status=status)
    assert status.tolist() == [0, 0, 0, fate.FATE_EINVAL]
    assert torch.equal(out[:73], good[:73])
    k = torch.randn(76, 2, 64).to(BF).cuda()
    status.zero_()
    fate.fate_attn_prompt(q.cuda(), k, k, torch.from_numpy(off2).cuda(), status=status)
    assert status.tolist() == [0, 0, 0, fate.FATE_EINVAL]


def test_on_another_stream_and_in_a_graph():
    args = make_paged([1, 1, 1], [900, 30, 2500], 8, 2, 128, BF, 16, seed=12)
    q, kc, vc, off, kv, pages = (t.cuda() for t in (*args[:3], *map(torch.from_numpy, args[3:])))
    want = ao.paged(*args[:3], args[3].tolist(), args[4].tolist(), args[5].tolist(), 1 / math.sqrt(128))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    out, lse = fate.fate_attn_paged(q, kc, vc, off, kv, pages, max_new=1, lse=True, stream=side)
    side.synchronize()
    compare(out, lse, want)
    # a captured step: the lengths are read on the device at each replay
    out = torch.empty_like(q)
    ws = torch.empty(fate.fate_attn_paged_ws_size(3, 8, kc, 3, pages.shape[1], 1), dtype=torch.uint8, device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        fate.fate_attn_paged(q, kc, vc, off, kv, pages, max_new=1, out=out, ws=ws)
    for lens in ([900, 30, 2500], [899, 1, 2000], [5, 30, 64], [900, 30, 2500]):
        kv.copy_(torch.tensor(lens, dtype=torch.int32))
        graph.replay()
        torch.cuda.synchronize()
        eager, _ = fate.fate_attn_paged(q, kc, vc, off, kv, pages, max_new=1)
        assert torch.equal(out, eager), lens
        q.copy_(torch.randn(q.shape, generator=torch.Generator().manual_seed(lens[0])).to(BF))


def test_empty_calls():
    z = torch.zeros(0, 4, 64, dtype=BF, device="cuda")
    c = torch.zeros(1, 4, 16, 64, dtype=BF, device="cuda")
    i = torch.zeros(1, dtype=torch.int32, device="cuda")
    out, lse = fate.fate_attn_prompt(z, z, z, i, lse=True)
    assert out.shape == (0, 4, 64) and lse.shape == (0, 4)
    none = torch.zeros(0, dtype=torch.int32, device="cuda")
    out, _ = fate.fate_attn_paged(z, c, c, i, none, torch.zeros(0, 1, dtype=torch.int32, device="cuda"))
    assert out.shape == (0, 4, 64)
    assert fate.fate_kv_append(z, z, z, c, c, i, none, torch.zeros(0, 1, dtype=torch.int32, device="cuda")).shape == (0, 4, 64)


def test_binding_refuses():
    args = make_paged([2], [20], 4, 2, 64, BF, 16)
    q, kc, vc, off, kv, pages = (t.cuda() for t in (*args[:3], *map(torch.from_numpy, args[3:])))
    ok = (q, kc, vc, off, kv, pages)

    def swap(i, t):
        return [*ok[:i], t, *ok[i + 1:]]

    for bad in (swap(0, q.float()), swap(0, q.half()), swap(0, q.cpu()), swap(0, q[0]), swap(0, q[..., :32]),
                swap(1, kc[:, :, :8]), swap(1, kc.half()), swap(2, vc.transpose(1, 2).contiguous().transpose(1, 2)),
                swap(3, off.long()), swap(4, kv.cpu()), swap(5, pages[0]), swap(4, kv[:0]),
                swap(0, q.transpose(1, 2).contiguous().transpose(1, 2))):
        with pytest.raises(ValueError):
            fate.fate_attn_paged(*bad)
    for more in (dict(scale=0.0), dict(scale=math.inf), dict(scale=-1.0), dict(scale=math.nan), dict(max_new=-1)):
        with pytest.raises(fate.FateError) as e:
            fate.fate_attn_paged(*ok, **more)
        assert e.value.status == fate.FATE_EINVAL
    with pytest.raises(fate.FateError) as e:
        fate.fate_attn_paged(*ok, ws=torch.empty(64, dtype=torch.uint8, device="cuda"))
    assert e.value.status == fate.FATE_ESIZE
    with pytest.raises(ValueError):
        fate.fate_attn_paged(*ok, status=torch.zeros(1, dtype=torch.int64, device="cuda"))
    odd = torch.zeros(2 * 4 * 64 + 1, dtype=BF, device="cuda")[1:].view(2, 4, 64)
    with pytest.raises(fate.FateError) as e:  # not aligned to 16 bytes
        fate.fate_attn_paged(*swap(0, odd))
    assert e.value.status == fate.FATE_EINVAL
    with pytest.raises(ValueError):
        fate.fate_kv_append(q, q[:, :2], q[:, :2].float(), kc, vc, off, kv, pages)
    with pytest.raises(ValueError):
        fate.fate_attn_prompt(q, q[:, :2], q[:1, :2], off)

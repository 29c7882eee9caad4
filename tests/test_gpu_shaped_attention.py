"""fate_attn_paged_shaped and fate_attn_prompt_shaped against attention in 64 bits: capped scores, bias by distance, first
keys (documents, windows) and prefixes.  Bounds are derived in serve_oracle.py from the kernels' arithmetic."""

import math

import numpy as np
import pytest
import torch

import attn_oracle as ao
import serve_oracle as so
from paper_2605_07238_amd import fate
from test_gpu_attention import BF, HEADS, HF, LENGTHS, compare, make_paged

pytestmark = pytest.mark.gpu


def shaping(kind, new, kv, hq, rng):
    """Arguments of a call of these lengths."""
    more, first = {}, []
    for n, L in zip(new, kv):
        pos = L - n + np.arange(n)
        if "document" in kind:
            cuts = np.concatenate([[0], np.cumsum(rng.integers(1, max(2, L // 3), 40))])
            first.append(cuts[np.searchsorted(cuts, np.maximum(pos, 0), side="right") - 1])
        elif "window" in kind:
            first.append(pos - [0, 5, 70, 300][len(first) % 4])  # also below 0; one key, some, many
        elif "nothing" in kind:  # rows whose first key lies past them: every other sequence, or its later rows
            first.append(np.where(np.arange(n) < (n // 2 if len(first) % 2 else 0), 0, np.maximum(pos, 0) + 1 + len(first)))
        else:
            first.append(np.zeros(n, int))
    if any(x in kind for x in ("document", "window", "nothing")):
        more["start"] = np.concatenate(first) if first else np.zeros(0)
    if "prefix" in kind:
        more["prefix"] = np.array([int(rng.integers(-2, L + 9)) if i % 3 else min(L, 64) for i, L in enumerate(kv)])
    if "cap" in kind:
        more["cap"] = 5000.0 if "wide" in kind else 3.0
    if "bias" in kind:
        more["slopes"] = np.array([2.0 ** (-8 * (h + 1) / hq) * (-0.01 if h % 5 == 4 else 1.0) for h in range(hq)], np.float32)
    return more


def on_gpu(more):
    kinds = dict(start=torch.int32, prefix=torch.int32, slopes=torch.float32)
    return {k: torch.as_tensor(np.ascontiguousarray(v), dtype=kinds[k]).cuda() if k in kinds else v for k, v in more.items()}


def expected(q, sequences, off, more, scale):
    """sequences: each one's keys and values [L, hkv, d]."""
    T, hq, d = q.shape
    unit, qd = ao.UNIT[q.dtype], q.double().numpy()
    out, lse = np.zeros((T, hq, d)), np.full((T, hq), -np.inf)
    tol, tol_lse = np.zeros((T, hq, d)), np.zeros((T, hq))
    for b, (keys, values) in enumerate(sequences):
        lo, hi = off[b], off[b + 1]
        if lo == hi:
            continue
        pos = len(keys) - (hi - lo) + np.arange(hi - lo)
        first = more["start"][lo:hi] if "start" in more else np.zeros(hi - lo)
        o, s, t, tl, w = so.attend_shaped(qd[lo:hi], keys, values, pos, more["prefix"][b] if "prefix" in more else 0, first, scale,
                                          more.get("cap", 0.0), more.get("slopes"))
        out[lo:hi], lse[lo:hi], tol[lo:hi], tol_lse[lo:hi] = o, s, ao.bound(t, o, w, unit), tl
    return out, lse, tol, tol_lse


def cached(kc, vc, kv, pages):
    P, got = kc.shape[2], []
    for b, L in enumerate(kv):
        at = np.arange(L)
        page, slot = pages[b][at // P] if L else at, at % P
        got.append([c.double().numpy()[page, :, slot] for c in (kc, vc)])
    return got


def run_paged(args, more, **rest):
    dev = [x.cuda() if isinstance(x, torch.Tensor) else torch.from_numpy(x).cuda() for x in args]
    return fate.fate_attn_paged_shaped(*dev, lse=True, **on_gpu(more), **rest)


KINDS = ["cap", "wide cap", "bias", "prefix", "document", "window", "nothing", "cap bias window", "bias prefix document",
         "nothing prefix", "cap prefix document", "wide cap bias prefix"]


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("lengths", range(len(LENGTHS)))
def test_paged(lengths, kind):
    new, kv = LENGTHS[lengths]
    which = lengths + KINDS.index(kind)
    heads, P, dtype = HEADS[which % len(HEADS)], [16, 1, 8, 64, 2, 32, 256][which // 2 % 7], BF if which % 2 else HF
    args = make_paged(new, kv, *heads, dtype, P, seed=which, scale_q=3.0)
    scale = 1 / math.sqrt(heads[2])
    more = shaping(kind, new, kv, heads[0], np.random.default_rng(which))
    want = expected(args[0], cached(*args[1:3], kv, args[5]), args[3], more, scale)
    for most in (max(new), None):
        status = torch.zeros(len(new), dtype=torch.int32, device="cuda")
        out, lse = run_paged(args, more, max_new=most, status=status)
        compare(out, lse, want)
        assert not status.any()


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("heads", [(8, 8, 64), (8, 2, 128), (5, 1, 256), (4, 2, 80), (7, 1, 16)], ids=str)
def test_prompt(heads, kind):
    hq, hkv, d = heads
    lens = [1, 64, 0, 65, 31, 127, 333, 2]
    which = KINDS.index(kind)
    dtype = BF if which % 2 else HF
    off = np.concatenate([[0], np.cumsum(lens)]).astype(np.int32)
    qkv = torch.randn(int(off[-1]), hq + 2 * hkv, d, generator=torch.Generator().manual_seed(which)).to(dtype)
    qkv[:, :hq] *= 3
    more = shaping(kind, lens, lens, hq, np.random.default_rng(which))
    sequences = [[qkv[lo:hi, a:b].double().numpy() for a, b in ((hq, hq + hkv), (hq + hkv, hq + 2 * hkv))]
                 for lo, hi in zip(off[:-1], off[1:])]
    want = expected(qkv[:, :hq], sequences, off, more, 1 / math.sqrt(d))
    x, status = qkv.cuda(), torch.zeros(len(lens), dtype=torch.int32, device="cuda")
    args = (x[:, :hq], x[:, hq:hq + hkv], x[:, hq + hkv:], torch.from_numpy(off).cuda())
    out, lse = fate.fate_attn_prompt_shaped(*args, lse=True, status=status, **on_gpu(more))
    compare(out, lse, want)
    assert not status.any()
    again, lse2 = fate.fate_attn_prompt_shaped(*args, lse=True, **on_gpu(more))
    assert torch.equal(out, again) and torch.equal(lse, lse2)


@pytest.mark.parametrize("kind", ["cap window", "bias prefix", "document prefix", "nothing"])
@pytest.mark.parametrize("new", [1, 4, 9, 40])
def test_split_axis(new, kind):
    """Long axes of different lengths, cut and joined, whole stretches of them unseen."""
    dtype = BF if new % 2 else HF
    lens = [new] * 4, [4099, 129, 9001, 6000]
    args = make_paged(*lens, 8, 2, 128, dtype, 16, seed=new, scale_q=2.0)
    more = shaping(kind, *lens, 8, np.random.default_rng(new))
    if "document" in kind:
        more["prefix"] = np.array([1000, 200, 3, 64])
    want = expected(args[0], cached(*args[1:3], args[4], args[5]), args[3], more, 0.1)
    out, lse = run_paged(args, more, max_new=new, scale=0.1)
    compare(out, lse, want)
    again, lse2 = run_paged(args, more, max_new=new, scale=0.1)
    assert torch.equal(out, again) and torch.equal(lse, lse2)


@pytest.mark.parametrize("most", [2, None])
def test_more_sequences_than_a_wave_has_lanes(most):
    rng = np.random.default_rng(0)
    new, kv = rng.integers(0, 3, 150).tolist(), rng.integers(2, 700, 150).tolist()
    args = make_paged(new, kv, 4, 2, 64, BF, 16, seed=0)
    more = shaping("bias prefix document", new, kv, 4, rng)
    want = expected(args[0], cached(*args[1:3], kv, args[5]), args[3], more, 0.125)
    compare(*run_paged(args, more, max_new=most), want)


@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
@pytest.mark.parametrize("n", [3, 200])
def test_unseen_keys_do_not_reach_a_row(n, bad):
    """Infinities and NaN in one document and between a prefix and a window reach those alone that see them."""
    for dtype in (BF, HF):
        args = make_paged([n], [n + 700], 4, 2, 128, dtype, 16, seed=n)
        q, kc, vc, off, kv, pages = args
        first = np.where(np.arange(n) < n // 2, 500, 700 + n // 2)  # the second document is of this call's rows alone
        more = dict(start=first, prefix=np.array([130]), cap=20.0)
        want = expected(q, cached(kc, vc, kv, pages), off, more, 1 / math.sqrt(128))
        for j in list(range(130, 500)) + [700 + n // 2 - 1]:  # seen by no row; by the last row of the first document
            for c in (kc, vc):
                c[int(pages[0, j // 16]), :, j % 16] = bad
        for most in (n, None):
            out, lse = run_paged(args, more, max_new=most)
            ok = np.arange(n) != n // 2 - 1
            compare(out[ok], lse[ok], [x[ok] for x in want])
            assert not torch.isfinite(out[n // 2 - 1]).any()


@pytest.mark.parametrize("n", [2, 150])
def test_infinite_values_in_a_seen_place(n):
    """A capped score is finite, so an infinite key does no harm by itself; an infinite value does to all who see it."""
    args = make_paged([n], [n + 100], 2, 1, 64, HF, 8, seed=n)
    q, kc, vc, off, kv, pages = args
    q[..., 0] = q[..., 0].abs() + 1
    kc[int(pages[0, 1]), :, 2, 0] = math.inf  # key 10
    more = dict(cap=4.0)
    clean = kc.clone()
    clean[int(pages[0, 1]), :, 2, 0] = 60000.0
    want = expected(q, cached(clean, vc, kv, pages), off, more, 0.125)
    compare(*run_paged(args, more, max_new=n), want)
    vc[int(pages[0, 1]), :, 2, 5] = math.inf
    out, _ = run_paged(args, more, max_new=n)
    assert torch.isinf(out[..., 5]).all() and torch.isfinite(out[..., :5]).all()


def test_first_keys_that_fall_are_reported():
    """In two tokens' rows of one workgroup, and of neighbouring ones; the other sequences are as they were."""
    for n, at in ((3, 2), (300, 16), (300, 17), (300, 128)):
        new, kv = [n, n, n], [n + 50] * 3
        args = make_paged(new, kv, 8, 1, 64, BF, 16, seed=n)
        start = np.tile(np.arange(n), 3)
        good = dict(start=start.copy())
        start[n + at] = at - 2
        for most in (n, None):
            status = torch.zeros(3, dtype=torch.int32, device="cuda")
            out, lse = run_paged(args, dict(start=start), max_new=most, status=status)
            assert status.tolist() == [0, -1, 0]
            want, lse2 = run_paged(args, good, max_new=most)
            keep = np.r_[0:n, 2 * n:3 * n]
            assert torch.equal(out[keep], want[keep]) and torch.equal(lse[keep], lse2[keep])
        x = args[0].cuda()
        status = torch.zeros(3, dtype=torch.int32, device="cuda")
        fate.fate_attn_prompt_shaped(x, x, x, torch.from_numpy(args[3]).cuda(), start=on_gpu(dict(start=start))["start"], status=status)
        assert status.tolist() == [0, -1, 0]
    # below 0 counts as 0, whatever the order
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    args = make_paged([3], [30], 8, 1, 64, BF, 16)
    run_paged(args, dict(start=np.array([-3, -7, -(1 << 31)])), status=status)
    assert not status.any()


def test_extreme_first_keys_and_prefixes():
    args = make_paged([3, 2], [30, 40], 4, 2, 64, BF, 16)
    big = (1 << 31) - 1
    for start, prefix in (([0, 0, big, big, big], [0, 0]), ([-(1 << 31)] * 5, [-(1 << 31), big]), ([29, 30, 31, 39, 39], [0, 1]),
                          ([big] * 5, [big, 0])):
        more = dict(start=np.array(start), prefix=np.array(prefix))
        want = expected(args[0], cached(*args[1:3], args[4], args[5]), args[3], more, 0.125)
        for most in (3, None):
            compare(*run_paged(args, more, max_new=most), want)


def test_as_the_plain_calls_without_shape():
    args = make_paged([5, 90, 1], [300, 90, 257], 8, 2, 128, HF, 16, seed=4)
    want = expected(args[0], cached(*args[1:3], args[4], args[5]), args[3], {}, 0.1)
    dev = [x.cuda() if isinstance(x, torch.Tensor) else torch.from_numpy(x).cuda() for x in args]
    for most in (5, 90, None):
        compare(*fate.fate_attn_paged(*dev, max_new=most, scale=0.1, lse=True), want)
        compare(*fate.fate_attn_paged_shaped(*dev, max_new=most, scale=0.1, lse=True), want)


def test_captured_with_other_masks_and_another_stream():
    """A captured call follows the arrays that shape it."""
    new, kv = [1, 2, 70], [300, 500, 900]
    args = make_paged(new, kv, 8, 2, 64, BF, 16, seed=2)
    dev = [x.cuda() if isinstance(x, torch.Tensor) else torch.from_numpy(x).cuda() for x in args]
    more = on_gpu(shaping("cap bias window prefix", new, kv, 8, np.random.default_rng(2)))
    out = torch.empty_like(dev[0])
    ws = torch.empty(fate.fate_attn_paged_ws_size(73, 8, dev[1], 3, dev[5].shape[1], 73), dtype=torch.uint8, device="cuda")
    go = lambda **x: fate.fate_attn_paged_shaped(*dev, max_new=73, **more, **x)[0]  # noqa: E731
    go(out=out, ws=ws)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    other = go(stream=side)
    side.synchronize()
    assert torch.equal(out, other)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        go(out=out, ws=ws)
    for step in range(4):
        more["start"] += 3
        more["prefix"] += 11
        more["slopes"] *= 0.5
        graph.replay()
        again = go()
        assert torch.equal(out, again)


def test_what_the_binding_refuses():
    args = make_paged([3], [30], 4, 2, 64, BF, 16)
    dev = [x.cuda() if isinstance(x, torch.Tensor) else torch.from_numpy(x).cuda() for x in args]
    good = on_gpu(dict(slopes=np.ones(4), prefix=np.array([3]), start=np.zeros(3)))
    prompt = (dev[0], dev[0], dev[0], dev[3])
    calls = (lambda **m: fate.fate_attn_paged_shaped(*dev, **dict(good, **m)),
             lambda **m: fate.fate_attn_prompt_shaped(*prompt, **dict(good, **m)))
    for call in calls:
        call()
        for name, bad in (("slopes", good["slopes"][:3]), ("slopes", good["slopes"].double()), ("prefix", good["prefix"].long()),
                          ("prefix", good["start"]), ("start", good["prefix"]), ("start", good["start"].cpu()),
                          ("start", torch.zeros(6, dtype=torch.int32, device="cuda")[::2])):
            with pytest.raises(ValueError):
                call(**{name: bad})
        for cap in (-1.0, math.inf, math.nan, 1e-44, 3e38):
            with pytest.raises(fate.FateError):
                call(cap=cap)
        with pytest.raises(ValueError, match="gradient"):
            call(slopes=good["slopes"].clone().requires_grad_())


@pytest.mark.parametrize("n", [3, 300])
def test_first_keys_that_fall_before_a_sequence_are_reported(n):
    """Rows that stand before their sequence (fewer keys than rows) see nothing, but where the first keys fall among them, or
    from them to the first that sees a key, the sequence is in error like any other; rows without a fall are not."""
    short = n - n // 3  # as many rows stand before the sequence
    new, kv = [n] * 3, [n + 50, n - short, n + 9]
    args = make_paged(new, kv, 8, 1, 64, BF, 16, seed=n)
    good = np.tile(np.arange(n), 3)
    for at in {1, short // 2, short - 1, short}:
        start = good.copy()
        start[n:n + at] = 1000
        for most in (n, None):
            status = torch.zeros(3, dtype=torch.int32, device="cuda")
            out, lse = run_paged(args, dict(start=start), max_new=most, status=status)
            assert status.tolist() == [0, -1, 0], (at, most)
            want, lse2 = run_paged(args, dict(start=good), max_new=most, status=status.zero_())
            assert not status.any()
            keep = np.r_[0:n, 2 * n:3 * n]
            assert torch.equal(out[keep], want[keep]) and torch.equal(lse[keep], lse2[keep])
    # below 0 counts as 0 here too, and none of it is looked at across sequences
    start = good.copy()
    start[n:n + short] = np.arange(short)[::-1] - 2 * n
    for most in (n, None):
        status = torch.zeros(3, dtype=torch.int32, device="cuda")
        compare(*run_paged(args, dict(start=start), max_new=most, status=status),
                expected(args[0], cached(*args[1:3], kv, args[5]), args[3], dict(start=start), 1 / math.sqrt(64)))
        assert not status.any()

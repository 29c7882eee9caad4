"""Kernel instances that other tests' sizes do not reach: appends larger than the last-level cache, pages of two and four
tokens, prompts and chunks of many key tiles, heads that fill a tile in part."""

import math

import numpy as np
import pytest
import torch

import attn_oracle as ao
from paper_2605_07238_amd import fate
from test_gpu_attention import BF, HF, compare, make_paged, run_paged

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [BF, HF], ids=["bf16", "f16"])
@pytest.mark.parametrize("rot,interleaved", [(256, False), (64, False), (128, True), (0, False)])
def test_append_past_the_last_level_cache(rot, interleaved, dtype):
    hq, hkv, d, P = 8, 8, 256, 16
    new, old = [5000, 1, 3007, 0, 4000], [3, 700, 0, 5, 129]
    T, half = sum(new), rot // 2
    assert T * (2 * hq + 4 * hkv) * d * 2 > 256 << 20  # the size from which rows are read past the cache
    off = np.concatenate([[0], np.cumsum(new)])
    kv = [a + b for a, b in zip(new, old)]
    gen = torch.Generator(device="cuda").manual_seed(rot)
    qkv = torch.randn(T, hq + 2 * hkv, d, generator=gen, device="cuda").to(dtype)
    need = [-(-n // P) for n in kv]
    order = torch.randperm(sum(need), generator=torch.Generator().manual_seed(1)).int()
    tables = torch.full((len(new), max(need)), -1, dtype=torch.int32)
    at = 0
    for b, n in enumerate(need):
        tables[b, :n] = order[at:at + n]
        at += n
    tables = tables.cuda()
    kc, vc = (torch.full((sum(need), hkv, P, d), 7.0, dtype=dtype, device="cuda") for _ in range(2))
    want_k, want_v = kc.clone(), vc.clone()
    table = fate.rotation_table(max(kv), rot) if rot else None
    status = torch.zeros(len(new), dtype=torch.int32, device="cuda")
    ints = lambda x: torch.tensor(list(map(int, x)), dtype=torch.int32, device="cuda")  # noqa: E731
    got = fate.fate_kv_append(qkv[:, :hq], qkv[:, hq:hq + hkv], qkv[:, hq + hkv:], kc, vc, ints(off), ints(kv), tables, table,
                              interleaved=interleaved, status=status)
    assert not status.any()
    seq = torch.repeat_interleave(torch.arange(len(new), device="cuda"), torch.tensor(new, device="cuda"))
    pos = torch.arange(T, device="cuda") - torch.tensor(off[:-1], device="cuda")[seq] + torch.tensor(old, device="cuda")[seq]
    page, slot = tables[seq, pos // P].long(), pos % P

    def close(x, y):
        """x: as computed, y: what went in."""
        y, bound = y.double(), torch.zeros(y.shape, dtype=torch.float64, device="cuda")
        want = y.clone()
        if rot:
            one, two = (slice(0, rot, 2), slice(1, rot, 2)) if interleaved else (slice(0, half), slice(half, rot))
            c, s = table.double()[pos][:, None, :half], table.double()[pos][:, None, half:]
            want[..., one], want[..., two] = y[..., one] * c - y[..., two] * s, y[..., two] * c + y[..., one] * s
            err = 2.0 ** -22 * (y[..., one].abs() + y[..., two].abs())
            for part in (one, two):
                bound[..., part] = err + ao.UNIT[dtype] * (want[..., part].abs() + err) + ao.TINY
        assert ((x.double() - want).abs() <= bound).all()

    close(got, qkv[:, :hq])
    close(kc[page, :, slot], qkv[:, hq:hq + hkv])
    assert torch.equal(vc[page, :, slot], qkv[:, hq + hkv:])
    # every other slot is as it was
    for c, want in ((kc, want_k), (vc, want_v)):
        want[page, :, slot] = c[page, :, slot]
        assert torch.equal(c, want)


@pytest.mark.parametrize("P", [1, 2, 4, 8])
@pytest.mark.parametrize("heads", [(4, 4, 64), (8, 2, 128), (2, 1, 256), (4, 2, 40), (2, 2, 200)], ids=str)
def test_small_pages(heads, P):
    new, kv = [70, 1, 130, 33], [200, 66, 131, 515]
    args = make_paged(new, kv, *heads, BF if P % 4 else HF, P, seed=P)
    scale = 1 / math.sqrt(heads[2])
    want = ao.paged(*args[:3], args[3].tolist(), args[4].tolist(), args[5].tolist(), scale)
    status = torch.zeros(4, dtype=torch.int32, device="cuda")
    compare(*run_paged(*args, max_new=130, status=status), want)
    assert not status.any()


@pytest.mark.parametrize("heads", [(2, 1, 128), (2, 2, 64), (1, 1, 256), (3, 1, 88)], ids=str)
@pytest.mark.parametrize("dtype", [BF, HF], ids=["bf16", "f16"])
def test_prompts_of_many_tiles(heads, dtype):
    hq, hkv, d = heads
    off = [0, 1537, 1537, 1600, 2611]
    gen = torch.Generator().manual_seed(d)
    q, k, v = (torch.randn(off[-1], h, d, generator=gen).to(dtype) for h in (hq, hkv, hkv))
    out, lse = fate.fate_attn_prompt(q.cuda(), k.cuda(), v.cuda(), torch.tensor(off, dtype=torch.int32, device="cuda"), lse=True)
    compare(out, lse, ao.prompt(q, k, v, off, 1 / math.sqrt(d)))


@pytest.mark.parametrize("bad", [math.nan, math.inf])
@pytest.mark.parametrize("P,d", [(2, 64), (16, 256), (4, 128)])
def test_unseen_values_over_parts(bad, P, d):
    """Infinite and NaN values at the last positions of chunks whose keys are walked in parts."""
    new, kv = [40, 35], [3000, 1200]
    args = make_paged(new, kv, 2, 1, d, HF, P, seed=d)
    q, kc, vc, off, lens, pages = args
    want = ao.paged(q, kc, vc, off.tolist(), lens.tolist(), pages.tolist(), 1 / math.sqrt(d))
    for b, L in enumerate(kv):
        for j in range(L - 10, L):
            for c in (kc, vc):
                c[int(pages[b, j // P]), :, j % P] = bad
    for most in (40, None):
        out, lse = run_paged(*args, max_new=most)
        for b in range(2):
            rows = slice(int(off[b]), int(off[b + 1]) - 10)
            compare(out[rows], lse[rows], [x[rows] for x in want])
            assert not torch.isfinite(out[int(off[b + 1]) - 10:int(off[b + 1])]).any()

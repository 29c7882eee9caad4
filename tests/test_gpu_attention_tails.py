"""A long flat tail of keys behind one large score: each key's weight is tiny, all of them together count."""

import numpy as np
import pytest
import torch

import attn_oracle as ao
from paper_2605_07238_amd import fate

pytestmark = pytest.mark.gpu

# Weights are rounded to the operands' type with the largest of a row at 2^7 or more (float16), so that one costs at most
# half a step of 2^-24 of them: 2^-32 of the largest.  Rounding of bfloat16, whose exponents reach further, is relative.
STEP = {torch.bfloat16: 0.0, torch.float16: 2.0 ** -32}


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16], ids=["bf16", "f16"])
@pytest.mark.parametrize("peak", [17.75, 15.5, 9.0])  # of the one key; the others' scores are zero
@pytest.mark.parametrize("n", [1, 40])
@pytest.mark.parametrize("where", ["first", "last"])
def test_flat_tail_behind_a_peak(dtype, peak, n, where):
    L, d, P = 100_000, 64, 64
    q = torch.zeros(n, 4, d, dtype=dtype)
    q[:, :, 0] = 4.0
    k = torch.zeros(L, 1, d, dtype=dtype)
    v = torch.ones(L, 1, d, dtype=dtype)
    at = 0 if where == "first" else L - n - 1  # seen by all rows
    k[at, 0, 0], v[at] = peak / 4, 0.0
    assert float(k[at, 0, 0]) * 4 == peak
    pages = -(-L // P)
    kc, vc = (torch.cat([x, x[:1].expand(pages * P - L, 1, d)]).view(pages, P, 1, d).transpose(1, 2).contiguous().cuda()
              for x in (k, v))
    one = lambda *x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    table = torch.arange(pages, dtype=torch.int32, device="cuda").view(1, -1)
    tail = (L - n + np.arange(n)).astype(float)  # keys of the tail that each row sees
    w = np.exp(-peak)
    want = tail * w / (1 + tail * w)
    unit = ao.UNIT[dtype]
    ds = (d + 2) * 2.0 ** -24 * peak + 2.0 ** -22 * (1 + peak)
    tol = (2 * ds + (L + 64) * 2.0 ** -24) * want + 2 * unit * want + STEP[dtype] * tail + ao.TINY
    for most in (n, None):
        out, lse = fate.fate_attn_paged(q.cuda(), kc, vc, one(0, n), one(L), table, max_new=most, scale=1.0, lse=True)
        assert (np.abs(out.double().cpu().numpy() - want[:, None, None]) <= tol[:, None, None]).all()
        assert np.allclose(lse.double().cpu().numpy(), (peak + np.log1p(tail * w))[:, None], atol=2 * ds + (L + 64) * 2.0 ** -24, rtol=0)
    if n == 1:  # as many answers as make a sequence one workgroup's, over the same pages
        B = 600
        off = torch.arange(B + 1, dtype=torch.int32, device="cuda")
        out, _ = fate.fate_attn_paged(q.cuda().expand(B, 4, d).contiguous(), kc, vc, off, one(*[L] * B), table.expand(B, -1),
                                      max_new=1, scale=1.0)
        assert (np.abs(out.double().cpu().numpy() - want[0]) <= tol[0]).all()
        return
    # a prompt of as many tokens: its last rows
    qs = torch.zeros(L, 4, d, dtype=dtype, device="cuda")
    qs[:, :, 0] = 4.0
    out, _ = fate.fate_attn_prompt(qs, k.cuda(), v.cuda(), one(0, L), scale=1.0)
    assert (np.abs(out[-n:].double().cpu().numpy() - want[:, None, None]) <= tol[:, None, None]).all()

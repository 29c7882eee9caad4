"""A serving step made of the device's calls alone: pages for the new tokens, rotation by several axes and the append,
shaped attention, the sampled token, and the keys that are given up again.  Each call is checked on what the calls before
it left, and a captured step against the eager one."""

import numpy as np
import pytest
import torch

import serve_oracle as so
from paper_2605_07238_amd import fate
from test_gpu_attention import compare
from test_gpu_shaped_attention import cached, expected

pytestmark = pytest.mark.gpu
HQ, HKV, D, P, WIDTH, N_PAGES, V, HIDDEN, WINDOW = 6, 2, 64, 16, 9, 40, 1031, 48, 37
SCALE, CAP = 0.125, 15.0
PROMPTS = [45, 1, 16, 30, 31]
B = len(PROMPTS)


def ints(x):
    return torch.as_tensor(np.ascontiguousarray(x), dtype=torch.int32).cuda()


class Serving:
    def __init__(self, dtype):
        gen = torch.Generator(device="cuda").manual_seed(5)
        rand = lambda *shape: torch.randn(*shape, generator=gen, device="cuda")  # noqa: E731
        self.embedding = rand(V, HIDDEN).to(dtype)
        self.weight = (rand(HIDDEN, (HQ + 2 * HKV) * D) / HIDDEN ** 0.5).to(dtype)
        self.last = (rand(HQ * D, V) / 8).to(dtype)
        self.slopes = torch.tensor([0.25 / (h + 1) for h in range(HQ)], device="cuda")
        self.table = fate.rotation_table(256, 48)
        self.axis = fate.rotation_axes((8, 8, 8))
        self.k, self.v = (torch.zeros(N_PAGES, HKV, P, D, dtype=dtype, device="cuda") for _ in range(2))
        self.pages = torch.full((B, WIDTH), -1, dtype=torch.int32, device="cuda")
        self.free, self.n_free = ints(np.random.default_rng(0).permutation(N_PAGES)), ints([N_PAGES])
        self.kv_len, self.new, self.drop = ints([0] * B), ints(PROMPTS), ints([0] * B)
        self.prefix = ints([4, 0, 3, 20, 1])
        self.tokens, self.status = ints([0] * B), ints([0] * B)
        self.u = torch.zeros(B, device="cuda")

    def state(self):
        return {k: x for k, x in vars(self).items() if isinstance(x, torch.Tensor)}

    def step(self, T, text=None, check=None):
        """One step of T rows: the prompts' tokens `text`, or each sequence's last token.  check(call, what it had, what it gave)."""
        told = check or (lambda *a: None)
        before = {k: x.clone() for k, x in self.state().items()} if check else None
        got = fate.Reserved(self.status.new_empty(B + 1), self.kv_len, self.n_free, self.status.new_empty(B + 1),
                            torch.empty(T, dtype=torch.int64, device="cuda"), self.status.new_empty(T))
        fate.fate_kv_reserve(self.new, self.kv_len, self.pages, self.free, self.n_free, P, T, out=got, status=self.status)
        told("reserve", before, got)
        row = torch.arange(T, device="cuda", dtype=torch.int32)
        of = torch.searchsorted(got.off[1:], row, right=True, out_int32=True).clamp(max=B - 1)
        x = self.embedding[(self.tokens[of] if text is None else text).long()]
        qkv = (x @ self.weight).view(T, HQ + 2 * HKV, D)
        at = got.positions.clamp(min=0)
        places = torch.stack([at, at // 7, at % 7]).int()
        q = fate.fate_kv_append_axes(qkv[:, :HQ], qkv[:, HQ:HQ + HKV], qkv[:, HQ + HKV:], self.k, self.v, got.off, self.kv_len, self.pages,
                                     self.table, places, self.axis, status=self.status)
        told("append", before, (got, qkv))
        shape = dict(scale=SCALE, cap=CAP, slopes=self.slopes, prefix=self.prefix, start=(got.positions - (WINDOW - 1)).int(), lse=True)
        if text is None:
            out, lse = fate.fate_attn_paged_shaped(q, self.k, self.v, got.off, self.kv_len, self.pages, max_new=1, **shape)
        else:  # the keys as the cache has them
            page, slot = got.slots // P, got.slots % P
            out, lse = fate.fate_attn_prompt_shaped(q, self.k[page, :, slot], self.v[page, :, slot], got.off, **shape)
        told("attention", before, (got, q, out, lse))
        ends = (got.off[1:] - 1).clamp(min=0).long()
        logits = out.flatten(1)[ends] @ self.last
        token, share = fate.fate_sample(logits, self.u, 0.8, top_k=50, top_p=0.95, min_p=0.001, logprob=True)
        told("sample", before, (logits, token, share))
        self.tokens.copy_(torch.where(self.new > 0, token, self.tokens))
        keep = (self.kv_len - self.drop).clamp(min=0)
        told("trim before", before, keep)
        cut = fate.Trimmed(self.kv_len, self.n_free, self.status.new_empty(B + 1))
        fate.fate_kv_trim(keep, self.kv_len, self.pages, self.free, self.n_free, P, out=cut, status=self.status)
        told("trim", before, (keep, cut))


def checks(s, T):
    """Checks of one step's calls; the cache and tables as they stand when a call has been made."""
    kept = {}
    num = lambda x: x.cpu().numpy()  # noqa: E731

    def check(call, before, got):
        if call == "reserve":
            want = so.reserve(num(before["new"]).tolist(), num(before["kv_len"]).tolist(), num(before["pages"]), num(before["free"]).tolist(),
                              int(before["n_free"]), P, T)
            for name, g, w in zip(got._fields + ("pages", "status"), tuple(got) + (s.pages, s.status), want):
                assert np.array_equal(num(g), w), name
        elif call == "append":
            res, qkv = got
            slots, kept["off"] = num(res.slots), num(res.off)
            rows = np.flatnonzero(slots >= 0)
            assert len(rows) == kept["off"][-1]
            page, slot = slots[rows] // P, slots[rows] % P
            for now, was, first in ((s.k, before["k"], HQ), (s.v, before["v"], HQ + HKV)):
                others = torch.ones(N_PAGES, P, dtype=torch.bool)
                others[page, slot] = False
                assert torch.equal(now.cpu().transpose(1, 2)[others], was.cpu().transpose(1, 2)[others])
                mine = now.cpu()[page, :, slot]
                assert torch.equal(mine[..., 48:], qkv.cpu()[rows, first:first + HKV, 48:])
            assert torch.equal(s.v.cpu()[page, :, slot], qkv.cpu()[rows, HQ + HKV:])
        elif call == "attention":
            res, q, out, lse = got
            n = kept["off"][-1]
            seqs = cached(s.k.cpu(), s.v.cpu(), num(s.kv_len).tolist(), num(s.pages))
            more = dict(cap=CAP, slopes=num(s.slopes), prefix=num(s.prefix), start=num(res.positions) - (WINDOW - 1))
            compare(out[:n], lse[:n], [x[:n] for x in expected(q.cpu(), seqs, kept["off"], more, SCALE)])
        elif call == "sample":
            logits, token, share = got
            for b in range(B):
                want, its = so.sample(num(logits[b].double()), 0.800000011920929, 50, float(np.float32(0.95)), float(np.float32(0.001)),
                                      float(s.u[b]))
                assert token[b] == want and abs(float(share[b]) - its) <= 2.0 ** -23 * abs(its) + 2.0 ** -38
        elif call == "trim before":
            kept["before"] = [num(x).copy() for x in (got, s.kv_len, s.pages, s.free, s.n_free)]
        else:
            keep, kv, pages, free, n_free = kept["before"]
            want = so.trim(keep.tolist(), kv.tolist(), pages, free.tolist(), int(n_free[0]), P)
            for g, w in zip(tuple(got[1]) + (s.free, s.status), want):
                assert np.array_equal(num(g), w)

    return check


def plan(step):
    """Tokens new, and given up again, per sequence: one rests, one ends, some go back over a page's edge."""
    new, drop = [1] * B, [0] * B
    if step % 3 == 1:
        new[2] = 0
    if step >= 5:
        new[3] = 0
    if step == 5:
        drop[3] = 1000  # all of its pages go back
    if step == 4:
        drop[0] = 20
    if step == 7:
        drop[4] = 8
    return new, drop


def prompts(s, check=None):
    T = sum(PROMPTS)
    s.u.copy_(torch.tensor([0.1, 0.9, 0.4, 0.7, 0.3]))
    text = torch.randint(0, V, (T,), generator=torch.Generator().manual_seed(1)).cuda()
    s.step(T, text, check(s, T) if check else None)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16], ids=["bf16", "f16"])
def test_every_call_of_a_run(dtype):
    s = Serving(dtype)
    prompts(s, checks)
    rng = torch.Generator().manual_seed(2)
    for step in range(10):
        new, drop = plan(step)
        s.new.copy_(ints(new)), s.drop.copy_(ints(drop)), s.u.copy_(torch.rand(B, generator=rng))
        s.step(B, check=checks(s, B))
        assert not s.status.any()
    held = int((-(-s.kv_len // P)).sum())
    assert int(s.n_free) + held == N_PAGES and s.kv_len[3] == 0


def test_a_captured_step_is_the_eager_one():
    eager, s = Serving(torch.bfloat16), Serving(torch.bfloat16)
    prompts(eager), prompts(s)
    s.new.copy_(ints([1] * B))
    saved = {k: x.clone() for k, x in s.state().items()}
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        s.step(B)  # loads what the step calls
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        s.step(B)
    for k, x in s.state().items():
        x.copy_(saved[k])
    rng = torch.Generator().manual_seed(3)
    for step in range(10):
        new, drop = plan(step)
        for x in (eager, s):
            x.new.copy_(ints(new)), x.drop.copy_(ints(drop))
        u = torch.rand(B, generator=rng)
        eager.u.copy_(u), s.u.copy_(u)
        graph.replay()
        eager.step(B)
        torch.cuda.synchronize()
        for k, x in s.state().items():
            assert torch.equal(x, eager.state()[k]), (step, k)

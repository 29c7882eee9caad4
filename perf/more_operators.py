"""The calls around the attention of a planned wave: inputs, one pass, its work and its exact results.

A device that serves the stages of a wave makes, beside the attention calls themselves, these:

  reserve  fate_kv_reserve: pages for new tokens from the free ones, row offsets, slots and positions, from lengths
  trim     fate_kv_trim: sequences cut back to the keys that stay, their other pages free again
  axes     fate_kv_append_axes: the append whose rotation has positions on several axes (time, height, width)
  paged    fate_attn_paged_shaped: attention over pages, its scores capped by a tanh, with a bias that grows with
           distance, with a first key per row (documents, windows) and a prefix that every row sees
  prompt   fate_attn_prompt_shaped: the same over whole prompts
  sample   fate_sample: one token a row, by temperature, top-k, top-p and min-p, from a given random number
"""

import math
import random
from typing import NamedTuple

import numpy as np
import torch

own = False

# Heads of queries, heads of keys and values, head size.
HEADS = [(8, 8, 64), (32, 8, 128), (64, 8, 128), (28, 4, 128), (10, 2, 256), (20, 4, 80), (16, 1, 128)]
DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
# Padded scores of the largest listed attention case: a drawn one has no more.
MOST_SCORES = 32 * 16384 * 16384
# Logits of the largest listed sampling case.
MOST_LOGITS = 512 * 131072


def paging(name, op, B, new, kv, page, spare=1.0, spread=1):
    """new: (least, most) tokens that come (trim: that go) per sequence; kv: keys cached before; spare: free pages as a
    share of those that the call asks for (under 1: the last sequences get none)."""
    c = dict(op=op, B=B, new_lo=new[0], new_hi=new[1], kv_lo=kv[0], kv_hi=kv[1], page=page, spare=spare, spread=spread)
    return dict(c, name=name) if name else c


def axes(name, B, new, kv, heads, dtype, page, sections, cyclic=False, interleaved=False, spread=1):
    """sections: rotated pairs of each axis."""
    hq, hkv, d = heads
    c = dict(op="axes", B=B, new_lo=new[0], new_hi=new[1], kv_lo=kv[0], kv_hi=kv[1], hq=hq, hkv=hkv, d=d, dtype=dtype,
             page=page, sections="-".join(map(str, sections)), cyclic=cyclic, interleaved=interleaved, spread=spread)
    return dict(c, name=name) if name else c


def attention(name, op, B, new, kv, heads, dtype, page=0, **more):
    """cap: 0 for none.  bias: slopes by head.  prefix: (least, most) keys that all rows see.  document: (least, most)
    tokens of the documents that a sequence is made of.  window: keys that a row sees, itself among them."""
    hq, hkv, d = heads
    c = dict(op=op, B=B, new_lo=new[0], new_hi=new[1], kv_lo=kv[0], kv_hi=kv[1], hq=hq, hkv=hkv, d=d, dtype=dtype,
             page=page, cap=0.0, bias=False, prefix_lo=0, prefix_hi=0, doc_lo=0, doc_hi=0, window=0, lse=False, spread=1)
    c.update(more)
    return dict(c, name=name) if name else c


def sampling(name, rows, vocab, dtype, filters, temperature=(0.5, 1.2), banned=0.0, logprob=False, spread=1):
    """filters: names of those that rows have, or "mixed" for each row its own.  banned: share of tokens at -infinity."""
    c = dict(op="sample", rows=rows, vocab=vocab, dtype=dtype, filters=filters, t_lo=temperature[0], t_hi=temperature[1],
             banned=banned, logprob=logprob, spread=spread)
    return dict(c, name=name) if name else c


def listed():
    big = (32, 8, 128)
    return [
        # One step of 64 answers: one token each, every sixteenth of them takes a page.  Latency.
        paging("reserve_step", "reserve", 64, (1, 1), (128, 4096), 16),
        # A round of 500 requests on a cache nearly full: chunks behind what they have cached, the last find no page.
        paging("reserve_many", "reserve", 500, (1, 2048), (1, 8192), 16, spare=0.9),
        # Drafted tokens of 200 answers, refused in part, and answers that end: pages go back.
        paging("trim_many", "trim", 200, (1, 8192), (1, 8192), 16),
        # One step of 64 answers about images, past the images' positions.
        axes("axes_step", 64, (1, 1), (128, 4096), big, "bf16", 16, (16, 24, 24)),
        # Prompts with images in them, 128 to 4096 tokens, stored.
        axes("axes_prompts", 16, (128, 4096), (0, 0), big, "bf16", 16, (16, 24, 24), cyclic=True),
        # One step of 64 answers of a model with capped scores, a layer whose rows see a window of 4096 keys.
        attention("paged_window", "paged", 64, (1, 1), (128, 16384), big, "bf16", 16, cap=50.0, window=4096),
        # Chunks of new tokens over cached prefixes, scores biased by distance; the prefix is seen as a whole.
        attention("paged_bias", "paged", 16, (64, 1024), (128, 4096), (16, 16, 128), "f16", 32, bias=True,
                  prefix_lo=64, prefix_hi=2048, lse=True),
        # A wave's prompts, all scores capped.
        attention("prompt_cap", "prompt", 16, (128, 4096), (0, 0), big, "bf16", cap=30.0),
        # One long row of documents, each for itself, behind a common instruction.
        attention("prompt_documents", "prompt", 1, (16384, 16384), (0, 0), big, "bf16", prefix_lo=200, prefix_hi=200,
                  doc_lo=100, doc_hi=4000, lse=True),
        # One answer's next token: latency.
        sampling("sample_one", 1, 50001, "f32", "top_k top_p", logprob=True),
        # One step of 64 answers, each with its own settings; some tokens are not allowed.
        sampling("sample_step", 64, 131072, "f32", "mixed", banned=0.05, logprob=True),
        # Many short answers at once, the nucleus alone.
        sampling("sample_many", 512, 131072, "bf16", "top_p"),
    ]


def log_of(rng, lo, hi):
    return int(round(lo * (hi / lo) ** rng.random()))


def draw(rng):
    def span(lo, hi):
        a, b = sorted((log_of(rng, lo, hi), log_of(rng, lo, hi)))
        return a, b

    op = rng.choice(["reserve", "trim", "axes", "paged", "paged", "prompt", "sample", "sample"])
    heads, dtype, page = rng.choice(HEADS), rng.choice(["bf16", "f16"]), rng.choice([1, 8, 16, 32, 64, 256])
    spread = rng.randrange(1 << 20)
    if op in ("reserve", "trim"):
        B = log_of(rng, 1, 500)
        new = rng.choice([(1, 1), span(1, 64), span(1, 2048)]) if op == "reserve" else span(1, 8192)
        return paging(None, op, B, new, span(1, 8192), page, rng.choice([1.0, 1.0, 0.5, 2.0]), spread)
    if op == "axes":
        new, kv = rng.choice([(1, 1), span(1, 64), span(1, 4096)]), span(1, 4096)
        B = log_of(rng, 1, max(1, min(128, 32768 // new[1])))
        pairs = rng.choice([heads[2] // 2, heads[2] // 2, heads[2] // 4])
        first = rng.randrange(1, pairs // 2)
        second = rng.randrange(1, (pairs - first + 1) // 2 + 1)
        sections = rng.choice([(first, second, pairs - first - second), (first, pairs - first)])
        return axes(None, B, new, kv, heads, dtype, page, sections, rng.random() < 0.5, rng.random() < 0.3, spread)
    if op == "sample":
        vocab = log_of(rng, 1000, 200003)
        rows = log_of(rng, 1, max(1, min(512, MOST_LOGITS // vocab)))
        filters = rng.choice(["none", "top_k", "top_p", "min_p", "top_k top_p", "top_p min_p", "mixed", "mixed"])
        return sampling(None, rows, vocab, rng.choice(sorted(DTYPES)), filters, rng.choice([(0.3, 0.9), (0.7, 1.5)]),
                        rng.choice([0.0, 0.0, 0.05, 0.9]), rng.random() < 0.5, spread)
    kinds = rng.choice(["cap", "bias", "prefix", "document", "window", "cap window", "bias prefix", "cap document prefix"])
    more = dict(lse=rng.random() < 0.5, spread=spread)
    if "cap" in kinds:
        more["cap"] = rng.choice([20.0, 30.0, 50.0])
    if "bias" in kinds:
        more["bias"] = True
    if "prefix" in kinds:
        more["prefix_lo"], more["prefix_hi"] = span(1, 2048)
    if "document" in kinds:
        more["doc_lo"], more["doc_hi"] = span(16, 4096)
    if "window" in kinds:
        more["window"] = log_of(rng, 16, 8192)
    hq, d = heads[0], heads[2]
    if op == "paged":
        new = rng.choice([(1, 1), (1, 1), span(1, 8), span(1, 64), span(16, 2048)])
        kv = span(1, 65536 if new[1] == 1 else 16384)
        limit = min(64, (1 << 20) // (new[1] + kv[1]) * 8 // hq, MOST_SCORES // (hq * new[1] * (new[1] + kv[1])))
        return attention(None, op, log_of(rng, 1, max(1, limit)), new, kv, heads, dtype, page, **more)
    new = span(1, 16384)
    while hq * new[1] * new[1] * d > MOST_SCORES * 128:
        new = (min(new[0], new[1] // 2), new[1] // 2)
    B = log_of(rng, 1, max(1, min(64, MOST_SCORES * 128 // (hq * new[1] * new[1] * d), 65536 // new[1])))
    return attention(None, op, B, new, (0, 0), heads, dtype, **more)


def spread_over(n, lo, hi, rng):
    """n lengths, even over the logarithm of lo to hi, in no order."""
    if lo == hi:
        return [lo] * n
    got = [int(round(lo * (hi / lo) ** ((i + rng.random()) / n))) for i in range(n)]
    rng.shuffle(got)
    return got


class Lengths(NamedTuple):
    """Per sequence: tokens of the call, keys cached before it, keys that all rows see, first keys of the rows."""

    new: list
    old: list
    prefix: list
    first: list


def lengths(c):
    rng = random.Random(c["spread"])
    new = spread_over(c["B"], c["new_lo"], c["new_hi"], rng)
    old = spread_over(c["B"], c["kv_lo"], c["kv_hi"], rng)
    if c["op"] not in ("paged", "prompt"):
        return Lengths(new, old, [], [])
    prefix = spread_over(c["B"], c["prefix_lo"], c["prefix_hi"], rng) if c["prefix_hi"] else [0] * c["B"]
    first = []
    for n, o, x in zip(new, old, prefix):
        at = np.arange(o, o + n)
        if c["doc_hi"]:
            starts = [x]
            while starts[-1] < o + n:
                starts.append(starts[-1] + log_of(rng, c["doc_lo"], c["doc_hi"]))
            starts = np.array([0] + starts)
            first.append(starts[np.searchsorted(starts, at, side="right") - 1])
        else:
            first.append(np.maximum(0, at - c["window"] + 1) if c["window"] else np.zeros(n, np.int64))
    return Lengths(new, old, prefix, first)


def ints(values, dtype=torch.int32):
    return torch.tensor(values, dtype=dtype, device="cuda")


def normal(gen, dtype, *shape, scale=1.0):
    out = torch.empty(shape, dtype=dtype, device="cuda")
    flat = out.view(-1)
    for at in range(0, flat.numel(), 1 << 26):
        part = flat[at:at + (1 << 26)]
        part.copy_(torch.randn(part.numel(), generator=gen, device="cuda").mul_(scale))
    return out


def paged_tables(kv_len, P, rng, more=0):
    """A page table in no order for these lengths, -1 past each sequence's last page, and `more` other pages."""
    need = [-(-n // P) for n in kv_len]
    order = list(range(sum(need) + more))
    rng.shuffle(order)
    tables, at = [], 0
    for n in need:
        tables.append(order[at:at + n])
        at += n
    return tables, order[at:]


def padded(tables, width):
    return ints([t + [-1] * (width - len(t)) for t in tables])


def prepare(case, seed):
    c = case
    gen = torch.Generator(device="cuda").manual_seed(seed)
    rng = random.Random(seed)
    if c["op"] == "sample":
        return prepare_sample(c, gen, rng)
    if c["op"] in ("reserve", "trim"):
        return prepare_paging(c, rng)
    dtype, P = DTYPES[c["dtype"]], c["page"]
    new, old, prefix, first = lengths(c)
    T, B, hq, hkv, d = sum(new), c["B"], c["hq"], c["hkv"], c["d"]
    qkv = normal(gen, dtype, T, hq + 2 * hkv, d)
    off = [0]
    for n in new:
        off.append(off[-1] + n)
    s = dict(case=c, q=qkv[:, :hq], k=qkv[:, hq:hq + hkv], v=qkv[:, hq + hkv:], off=ints(off), max_new=max(new),
             scale=1.0 / math.sqrt(d))
    kv_len = [a + b for a, b in zip(old, new)]
    if c["op"] != "prompt":
        tables, _ = paged_tables(kv_len, P, rng)
        n_pages = sum(map(len, tables))
        s.update(kv_len=ints(kv_len), max_kv=max(kv_len), pages=padded(tables, max(map(len, tables))),
                 k_cache=normal(gen, dtype, n_pages, hkv, P, d), v_cache=normal(gen, dtype, n_pages, hkv, P, d))
    if c["op"] == "axes":
        sections = [int(x) for x in c["sections"].split("-")]
        half, n_axes = sum(sections), len(sections)
        angle = torch.outer(torch.arange(max(kv_len) + 1, dtype=torch.float64), 10000.0 ** (-torch.arange(half, dtype=torch.float64) / half))
        s["table"] = torch.cat([angle.cos(), angle.sin()], 1).float().cuda()
        s["axis"] = pair_axes(sections, c["cyclic"])
        # text stands at the same position on every axis; images of 16 x 24 patches at one time, row and column
        at = np.concatenate([np.arange(o, o + n) for o, n in zip(old, new)])
        inside, patch = (at // 512) % 2 == 1, at % 512 % 384
        base = at // 512 * 128
        where = [np.where(inside, base, at // 4), np.where(inside, base + patch // 24, at // 4),
                 np.where(inside, base + patch % 24, at // 4)]
        s["positions"] = ints(np.minimum(np.stack(where[:n_axes]), max(kv_len)))
        return s
    if c["op"] in ("paged", "prompt"):
        s["q"].mul_(4.0)  # scores of a trained model reach tens
        if c["bias"]:
            s["slopes"] = ints([2.0 ** (-8.0 * (h + 1) / hq) for h in range(hq)], torch.float32)
        if c["prefix_hi"]:
            s["prefix"] = ints(prefix)
        if c["doc_hi"] or c["window"]:
            s["start"] = ints(np.concatenate(first))
    return s


def pair_axes(sections, cyclic):
    """Each pair's axis: one section after the other, or in turn while a section has pairs left."""
    if not cyclic:
        return tuple(a for a, n in enumerate(sections) for _ in range(n))
    left, out = list(sections), []
    while any(left):
        for a in range(len(left)):
            if left[a]:
                left[a] -= 1
                out.append(a)
    return tuple(out)


def prepare_paging(c, rng):
    P, B = c["page"], c["B"]
    new, old, _, _ = lengths(c)
    more = 100
    if c["op"] == "reserve":
        more = int(sum(-(-(n + o) // P) - -(-o // P) for n, o in zip(new, old)) * c["spare"])
    tables, free = paged_tables(old, P, rng, more)
    held = sum(map(len, tables))
    s = dict(case=c, kv_len=ints(old), free=ints(free + [-1] * held), n_free=ints([len(free)]),
             status=torch.zeros(B, dtype=torch.int32, device="cuda"))
    if c["op"] == "reserve":
        s.update(new=ints(new), T=sum(new), pages=padded(tables, max(-(-(n + o) // P) for n, o in zip(new, old))))
    else:
        s.update(keep=ints([max(0, o - n) for n, o in zip(new, old)]), pages=padded(tables, max(map(len, tables))))
    return s


def prepare_sample(c, gen, rng):
    R, V = c["rows"], c["vocab"]
    logits = normal(gen, DTYPES[c["dtype"]], R, V, scale=2.5)
    # some thirty tokens of a row stand out, as they do in text
    some = torch.randint(0, V, (R, 32), generator=gen, device="cuda")
    logits.scatter_(1, some, (torch.randn(R, 32, generator=gen, device="cuda") * 2.5 + 9.0).to(logits.dtype))
    if c["banned"]:
        for r in range(R):
            logits[r].masked_fill_(torch.rand(V, generator=gen, device="cuda") < c["banned"], -math.inf)
    mixed = c["filters"] == "mixed"

    def some_of(name, values, none, dtype):
        if not mixed and name not in c["filters"].split():
            return None
        return ints([rng.choice(values + ([none] * len(values) if mixed else [])) for _ in range(R)], dtype)

    spread = [c["t_lo"] + (c["t_hi"] - c["t_lo"]) * rng.random() for _ in range(R)]
    if mixed:
        spread = [0.0 if rng.random() < 0.1 else t for t in spread]
    return dict(case=c, logits=logits, u=torch.rand(R, generator=gen, device="cuda"), temperature=ints(spread, torch.float32),
                top_k=some_of("top_k", [1, 20, 50, 200, 1000], 0, torch.int32),
                top_p=some_of("top_p", [0.5, 0.8, 0.9, 0.95, 0.99], 1.0, torch.float32),
                min_p=some_of("min_p", [0.01, 0.05, 0.1], 0.0, torch.float32))


def run(state):
    s, c = state, state["case"]
    if not own:
        return PLAIN[c["op"]](s)
    from paper_2605_07238_amd import fate
    if c["op"] == "reserve":
        got = fate.fate_kv_reserve(s["new"], s["kv_len"], s["pages"], s["free"], s["n_free"], c["page"], s["T"], status=s["status"])
        return got.off, got.kv_len, got.n_free, got.taken, got.slots, got.positions, s["pages"], s["status"]
    if c["op"] == "trim":
        got = fate.fate_kv_trim(s["keep"], s["kv_len"], s["pages"], s["free"], s["n_free"], c["page"], status=s["status"])
        return got.kv_len, got.n_free, got.given, s["free"], s["status"]
    if c["op"] == "axes":
        q = fate.fate_kv_append_axes(s["q"], s["k"], s["v"], s["k_cache"], s["v_cache"], s["off"], s["kv_len"], s["pages"],
                                     s["table"], s["positions"], s["axis"], interleaved=c["interleaved"])
        return q, s["k_cache"], s["v_cache"]
    if c["op"] == "sample":
        more = {k: s[k] for k in ("top_k", "top_p", "min_p") if s[k] is not None}
        token, logprob = fate.fate_sample(s["logits"], s["u"], temperature=s["temperature"], logprob=c["logprob"], **more)
        return (token, logprob) if c["logprob"] else (token,)
    more = dict(scale=s["scale"], cap=c["cap"], slopes=s.get("slopes"), prefix=s.get("prefix"), start=s.get("start"), lse=c["lse"])
    if c["op"] == "paged":
        out, lse = fate.fate_attn_paged_shaped(s["q"], s["k_cache"], s["v_cache"], s["off"], s["kv_len"], s["pages"],
                                               max_new=s["max_new"], **more)
    else:
        out, lse = fate.fate_attn_prompt_shaped(s["q"], s["k"], s["v"], s["off"], **more)
    return (out, lse) if c["lse"] else (out,)


def scan(x):
    """Sums before each element, and of all."""
    out = torch.zeros(x.shape[0] + 1, dtype=torch.int64, device=x.device)
    torch.cumsum(x, 0, out=out[1:])
    return out


def plain_reserve(s):
    P, pages = s["case"]["page"], s["pages"]
    new, old, n_free = s["new"].long(), s["kv_len"].long(), s["n_free"].long()
    have = (old + P - 1) // P
    need = (old + new + P - 1) // P - have
    fits = ((need == 0) | (scan(need)[1:] <= n_free)) & (scan(new)[1:] <= s["T"])
    new, need = new * fits, need * fits
    off, taken, kv = scan(new), scan(need), old + new
    j = torch.arange(pages.shape[1], device=pages.device) - have[:, None]
    page = s["free"][(n_free - 1 - taken[:-1, None] - j).clamp(0, s["free"].shape[0] - 1)]
    pages.copy_(torch.where((j >= 0) & (j < need[:, None]), page, pages))
    t = torch.arange(s["T"], device=pages.device)
    b = torch.searchsorted(off[1:].contiguous(), t, right=True).clamp(max=new.shape[0] - 1)
    pos = torch.where(t < off[-1], old[b] + t - off[b], -1)
    slots = torch.where(pos >= 0, pages[b, pos.clamp(min=0) // P].long() * P + pos % P, -1)
    return off.int(), kv.int(), (n_free - taken[-1:]).int(), taken.int(), slots, pos.int(), pages, torch.where(fits, 0, -5).int()


def plain_trim(s):
    P, pages, free = s["case"]["page"], s["pages"], s["free"]
    old, n_free = s["kv_len"].long(), s["n_free"].long()
    stay = torch.minimum(s["keep"].long(), old)
    have, left = (old + P - 1) // P, (stay + P - 1) // P
    gone = have - left
    fits = (gone == 0) | (n_free + scan(gone)[1:] <= free.shape[0])
    gone, kv = gone * fits, torch.where(fits, stay, old)
    given = scan(gone)
    j = torch.arange(pages.shape[1], device=pages.device) - left[:, None]
    to = torch.where((j >= 0) & (j < gone[:, None]), n_free + given[:-1, None] + j, free.shape[0])
    free.copy_(torch.cat([free, free[:1]]).scatter_(0, to.flatten(), pages.flatten())[:-1])
    return kv.int(), (n_free + given[-1:]).int(), given.int(), free, torch.where(fits, 0, -1).int()


def rows_of(off, T):
    """Each token's sequence and its place among that sequence's tokens."""
    t = torch.arange(T, device=off.device)
    b = torch.searchsorted(off[1:].long().contiguous(), t, right=True)
    return b, t - off.long()[b]


def plain_axes(s):
    c = s["case"]
    b, i = rows_of(s["off"], s["q"].shape[0])
    slot = (s["kv_len"].long() - (s["off"][1:] - s["off"][:-1]).long())[b] + i
    half = len(s["axis"])
    turn = s["positions"][torch.tensor(s["axis"], device=slot.device)].long().t()  # [T, half]
    pair = torch.arange(half, device=slot.device)
    cos, sin = s["table"][turn, pair][:, None], s["table"][turn, half + pair][:, None]

    def rotated(x):
        y = x.float()
        one, two = (y[..., 0:2 * half:2], y[..., 1:2 * half:2]) if c["interleaved"] else (y[..., :half], y[..., half:2 * half])
        u, w = one * cos - two * sin, two * cos + one * sin
        turned = torch.stack([u, w], -1).flatten(-2) if c["interleaved"] else torch.cat([u, w], -1)
        return torch.cat([turned, y[..., 2 * half:]], -1).to(x.dtype)

    page, slot = s["pages"][b, slot // c["page"]].long(), slot % c["page"]
    s["k_cache"][page, :, slot] = rotated(s["k"])
    s["v_cache"][page, :, slot] = s["v"]
    return rotated(s["q"]), s["k_cache"], s["v_cache"]


def softmax_product(s, q, k, v, b, i, old, n_kv):
    """q (B, n, heads_q, d) over k and v (B, L, heads_kv, d); rows b, i of these are the call's, at position old[b] + i."""
    c = s["case"]
    B, n, hq, d = q.shape
    L, hkv = k.shape[1], k.shape[2]
    j, p = torch.arange(L, device=q.device), old[:, None] + torch.arange(n, device=q.device)
    first = torch.zeros((B, n), dtype=torch.int64, device=q.device)
    if "start" in s:
        first[b, i] = s["start"].long()
    seen = (j <= p[..., None]) & (j >= first[..., None])
    if "prefix" in s:
        seen |= j < torch.minimum(s["prefix"].long(), n_kv)[:, None, None]
    q = q.float().reshape(B, n, hkv, hq // hkv, d).permute(0, 2, 3, 1, 4).reshape(B * hkv, -1, d)
    kt = k.float().permute(0, 2, 3, 1).reshape(B * hkv, d, L)
    sc = torch.bmm(q, kt).mul_(s["scale"]).view(B, hkv, hq // hkv, n, L)
    if c["cap"]:
        sc.div_(c["cap"]).tanh_().mul_(c["cap"])
    if c["bias"]:
        sc.addcmul_(s["slopes"].view(1, hkv, hq // hkv, 1, 1), (p[..., None] - j).abs().float()[:, None, None], value=-1.0)
    sc.masked_fill_(~seen[:, None, None], -math.inf)
    top = sc.amax(-1, keepdim=True).clamp_(min=-3e38)
    sc.sub_(top).exp_()
    total = sc.sum(-1, keepdim=True)
    out = torch.bmm(sc.view(B * hkv, -1, L), v.float().permute(0, 2, 1, 3).reshape(B * hkv, L, d)).view(B, hkv, hq // hkv, n, d)
    out = (out / total.clamp(min=1e-38)).permute(0, 3, 1, 2, 4).reshape(B, n, hq, d)[b, i].to(s["q"].dtype)
    lse = (top + total.log())[..., 0].permute(0, 3, 1, 2).reshape(B, n, hq)[b, i]
    return (out, lse) if c["lse"] else (out,)


def plain_paged(s):
    c, off = s["case"], s["off"].long()
    b, i = rows_of(s["off"], s["q"].shape[0])
    at = (off[:-1, None] + torch.arange(s["max_new"], device=off.device)).clamp(max=s["q"].shape[0] - 1)
    j = torch.arange(s["max_kv"], device=off.device)
    page, slot = s["pages"][:, j // c["page"]].long().clamp(min=0), j % c["page"]
    n_kv = s["kv_len"].long()
    return softmax_product(s, s["q"][at], s["k_cache"][page, :, slot], s["v_cache"][page, :, slot], b, i,
                           n_kv - (off[1:] - off[:-1]), n_kv)


def plain_prompt(s):
    off = s["off"].long()
    b, i = rows_of(s["off"], s["q"].shape[0])
    at = (off[:-1, None] + torch.arange(s["max_new"], device=off.device)).clamp(max=s["q"].shape[0] - 1)
    n_kv = off[1:] - off[:-1]
    return softmax_product(s, s["q"][at], s["k"][at], s["v"][at], b, i, torch.zeros_like(n_kv), n_kv)


def plain_sample(s):
    """In 64 bits: whole numbers that hang on long sums and on values next to a border."""
    logits, t = s["logits"], s["temperature"].double()[:, None]
    R, V = logits.shape
    k = s["top_k"].long()[:, None] if s["top_k"] is not None else torch.zeros_like(t, dtype=torch.int64)
    k = torch.where(t == 0, 1, torch.where(k == 0, V, k))
    value, order = torch.sort(logits.double(), dim=-1, descending=True, stable=True)
    w = ((value - value[:, :1]) / torch.where(t == 0, 1.0, t)).exp()
    w = w * (torch.arange(V, device=w.device) < k)
    if s["top_p"] is not None:
        p, before = s["top_p"].double()[:, None], w.cumsum(-1) - w
        w = w * ((before < p * w.sum(-1, keepdim=True)) | (p >= 1))
    if s["min_p"] is not None:
        w = w * (w >= s["min_p"].double()[:, None])
    w = torch.zeros_like(w).scatter_(1, order, w)
    upto = w.cumsum(-1)
    token = (upto <= s["u"].double()[:, None] * upto[:, -1:]).sum(-1)
    if not s["case"]["logprob"]:
        return (token.int(),)
    return token.int(), (w.gather(1, token[:, None])[:, 0] / upto[:, -1]).log().float()


PLAIN = {"reserve": plain_reserve, "trim": plain_trim, "axes": plain_axes, "paged": plain_paged, "prompt": plain_prompt,
         "sample": plain_sample}


def work(case):
    c = case
    if c["op"] == "sample":
        e = 4 if c["dtype"] == "f32" else 2
        # a sum, or a comparison, of each logit
        return {"bytes": c["rows"] * (c["vocab"] * e + 16), "flops": 2 * c["rows"] * c["vocab"]}
    new, old, prefix, first = lengths(c)
    T, e, B, P = sum(new), 2, c["B"], c["page"]
    if c["op"] in ("reserve", "trim"):
        if c["op"] == "reserve":
            moved = sum(-(-(n + o) // P) - -(-o // P) for n, o in zip(new, old))
        else:
            moved = sum(-(-o // P) - -(-max(0, o - n) // P) for n, o in zip(new, old))
        return {"bytes": B * 24 + moved * 8 + (T * 12 if c["op"] == "reserve" else 0), "flops": 0}
    if c["op"] == "axes":
        half = sum(int(x) for x in c["sections"].split("-"))
        n_axes = c["sections"].count("-") + 1
        return {"bytes": T * ((2 * c["hq"] + 4 * c["hkv"]) * c["d"] * e + 4 * n_axes) + (max(map(max, (old, new))) * half * 8), "flops": 0}
    pairs = keys = 0
    for n, o, x, f in zip(new, old, prefix, first):
        p, x = np.arange(o, o + n), min(x, o + n)
        pairs += int((x + np.maximum(0, p + 1 - np.maximum(f, x))).sum())
        keys += x + max(0, o + n - max(x, int(f[0])))
    rows = T * (c["hq"] * (2 * c["d"] * e + (4 if c["lse"] else 0)) + (4 if c["doc_hi"] or c["window"] else 0))
    return {"bytes": rows + keys * 2 * c["hkv"] * c["d"] * e, "flops": 4 * c["hq"] * c["d"] * pairs}


def exact(case, seed):
    """From the definitions, sequence by sequence and row by row; computed numbers in 64 bits."""
    c = case
    s = prepare(c, seed)
    if c["op"] == "reserve":
        return exact_reserve(c, s)
    if c["op"] == "trim":
        return exact_trim(c, s)
    if c["op"] == "sample":
        return exact_sample(c, s)
    off = s["off"].tolist()
    if c["op"] == "axes":
        return exact_axes(c, s, off)
    G, P = c["hq"] // c["hkv"], c["page"]
    out = torch.empty(s["q"].shape, dtype=torch.float64, device="cuda")
    lse = torch.empty(s["q"].shape[:2], dtype=torch.float64, device="cuda")
    _, _, prefix, first = lengths(c)
    for b in range(c["B"]):
        lo, hi = off[b], off[b + 1]
        if c["op"] == "paged":
            n_kv = s["kv_len"].tolist()[b]
            ids = s["pages"][b, :-(-n_kv // P)].long()
            keys, values = (x[ids].double().transpose(1, 2).flatten(0, 1)[:n_kv] for x in (s["k_cache"], s["v_cache"]))
        else:
            n_kv = hi - lo
            keys, values = s["k"][lo:hi].double(), s["v"][lo:hi].double()
        j = torch.arange(n_kv, device="cuda")
        step = max(1, (1 << 27) // max(1, n_kv * G))
        for h in range(c["hkv"]):
            kh, vh = keys[:, h].t().contiguous(), values[:, h].contiguous()
            for at in range(lo, hi, step):
                end = min(hi, at + step)
                pos = n_kv - (hi - lo) + (at - lo) + torch.arange(end - at, device="cuda")
                begin = torch.from_numpy(np.asarray(first[b][at - lo:end - lo])).cuda()
                hidden = ((j > pos[:, None]) | (j < begin[:, None])) & (j >= prefix[b])
                rows = s["q"][at:end, h * G:(h + 1) * G].double().reshape(-1, c["d"])
                sc = ((rows @ kh) * s["scale"]).view(end - at, G, n_kv)
                if c["cap"]:
                    sc = c["cap"] * torch.tanh(sc / c["cap"])
                if c["bias"]:
                    sc -= s["slopes"][h * G:(h + 1) * G].double()[:, None] * (pos[:, None, None] - j).abs()
                sc = sc.masked_fill(hidden[:, None], -math.inf)
                l = torch.logsumexp(sc, 2)
                out[at:end, h * G:(h + 1) * G] = torch.exp(sc - l[..., None]) @ vh
                lse[at:end, h * G:(h + 1) * G] = l
    return (out, lse) if c["lse"] else (out,)


def exact_reserve(c, s):
    P, T = c["page"], s["T"]
    new, kv, pages, free = s["new"].tolist(), s["kv_len"].tolist(), s["pages"].tolist(), s["free"].tolist()
    n_free = s["n_free"].item()
    asked = tokens = given = 0
    off, taken, slots, positions, status = [0], [0], [], [], []
    for b in range(c["B"]):
        more = -(-(kv[b] + new[b]) // P) - -(-kv[b] // P)
        asked, tokens = asked + more, tokens + new[b]
        ok = (more == 0 or asked <= n_free) and tokens <= T
        status.append(0 if ok else -5)
        if ok:
            for x in range(more):
                pages[b][-(-kv[b] // P) + x] = free[n_free - 1 - given - x]
            given += more
            for at in range(kv[b], kv[b] + new[b]):
                positions.append(at)
                slots.append(pages[b][at // P] * P + at % P)
            kv[b] += new[b]
        off.append(len(positions))
        taken.append(given)
    rest = [-1] * (T - len(slots))
    return ints(off), ints(kv), ints([n_free - given]), ints(taken), ints(slots + rest, torch.int64), ints(positions + rest), ints(pages), ints(status)


def exact_trim(c, s):
    P, keep, kv, pages, free = c["page"], s["keep"].tolist(), s["kv_len"].tolist(), s["pages"].tolist(), s["free"].tolist()
    n_free = s["n_free"].item()
    given, total = [0], 0
    for b in range(c["B"]):
        stay = min(keep[b], kv[b])
        for page in pages[b][-(-stay // P):-(-kv[b] // P)]:
            free[n_free + total] = page
            total += 1
        kv[b] = stay
        given.append(total)
    return ints(kv), ints([n_free + total]), ints(given), ints(free), torch.zeros_like(s["status"])


def exact_axes(c, s, off):
    kv_len, tables, P, half = s["kv_len"].tolist(), s["pages"].tolist(), c["page"], len(s["axis"])
    q, kc, vc, new_k = s["q"].double(), s["k_cache"].double(), s["v_cache"].double(), s["k"].double()
    first, second = (slice(0, 2 * half, 2), slice(1, 2 * half, 2)) if c["interleaved"] else (slice(0, half), slice(half, 2 * half))
    turn = torch.empty((q.shape[0], 1, half), dtype=torch.complex128, device="cuda")
    for i, a in enumerate(s["axis"]):
        at = s["positions"][a].long()
        turn[:, 0, i] = torch.complex(s["table"][at, i].double(), s["table"][at, half + i].double())
    for x in (q, new_k):
        z = torch.complex(x[..., first].clone(), x[..., second].clone()) * turn
        x[..., first], x[..., second] = z.real, z.imag
    for b in range(c["B"]):
        lo, hi = off[b], off[b + 1]
        where = torch.tensor([tables[b][p // P] * P + p % P for p in range(kv_len[b] - (hi - lo), kv_len[b])], device="cuda")
        for cache, x in ((kc, new_k), (vc, s["v"].double())):
            for h in range(c["hkv"]):
                cache[where // P, h, where % P] = x[lo:hi, h]
    return q, kc, vc


def exact_sample(c, s):
    tokens, logprobs = [], []
    settings = [x.tolist() if x is not None else [none] * c["rows"] for x, none in (
        (s["temperature"], None), (s["top_k"], 0), (s["top_p"], 1.0), (s["min_p"], 0.0), (s["u"], None))]
    for r, (t, k, p, least, u) in enumerate(zip(*settings)):
        row = s["logits"][r].double()
        if t == 0.0:
            tokens.append((row == row.max()).nonzero()[0, 0])
            logprobs.append(torch.zeros((), dtype=torch.float64, device="cuda"))
            continue
        prob = torch.softmax(row / t, 0)
        ranked = torch.argsort(-row, stable=True)
        if k:
            ranked = ranked[:k]
        among = prob[ranked] / prob[ranked].sum()
        keep = torch.ones_like(ranked, dtype=torch.bool)
        if p < 1:
            total = among.cumsum(0)
            keep[1:] = total[:-1] < p  # the tokens above it fall short of p
        ranked = ranked[keep & (among >= least * among[0])]
        at = ranked.sort().values
        share = prob[at] / prob[at].sum()
        i = torch.searchsorted(share.cumsum(0), torch.tensor([u], dtype=torch.float64, device="cuda"), right=True).clamp(max=at.numel() - 1)[0]
        tokens.append(at[i])
        logprobs.append(share[i].log())
    token = torch.stack(tokens).int()
    return (token, torch.stack(logprobs)) if c["logprob"] else (token,)

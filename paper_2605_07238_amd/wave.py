"""A planned wave, carried out: the attention calls that one device makes for
the stages that the planner gave it.

The planner (score, top-k, planning wave, commit; :mod:`.fate`) says which
stages run on a device next and, through its prefix slots, which prompts start
with a prefix whose keys and values the device still holds.  :class:`DeviceCache`
is what such a slot stands for on the device: pages of a paged cache per workflow,
model and prefix group.  :func:`carry_out` lets go of the groups that the plan's
slots no longer name and gives each device its stages; :func:`run_stages` takes
those of one model through one attention layer:

  stages whose prefix is cached   their own tokens are appended behind the
                                  shared pages and attend over them
                                  (fate_kv_append, fate_attn_paged)
  the others                      the whole prompt is attended and stored
                                  (fate_kv_append, fate_attn_prompt), and the
                                  prefix's full pages become the group's
  then all of them                answer token by token (fate_kv_append,
                                  fate_attn_paged)

``python -m paper_2605_07238_amd.wave`` plans waves on a few fork-join
workflows, carries out each device's share and prints per wave the time with
cached prefixes and without.  Weights and tokens are random.
"""

from __future__ import annotations

import dataclasses
import time

import numpy as np
import torch

from . import fate, synth


@dataclasses.dataclass
class Layer:
    """One attention layer: heads, the fused projection and the rotation table."""

    heads_q: int
    heads_kv: int
    head_dim: int
    weight: torch.Tensor  # [hidden, (heads_q + 2 heads_kv) head_dim]
    table: torch.Tensor   # [positions, head_dim]

    @classmethod
    def random(cls, hidden=512, heads_q=32, heads_kv=8, head_dim=128, positions=8192, dtype=torch.bfloat16, seed=0):
        gen = torch.Generator(device="cuda").manual_seed(seed)
        weight = torch.randn(hidden, (heads_q + 2 * heads_kv) * head_dim, generator=gen, device="cuda") / hidden ** 0.5
        return cls(heads_q, heads_kv, head_dim, weight.to(dtype), fate.rotation_table(positions, head_dim))

    def project(self, x):
        """Fused projection [T, heads_q + 2 heads_kv, head_dim] of token rows x [T, hidden]."""
        return (x @ self.weight).view(x.shape[0], self.heads_q + 2 * self.heads_kv, self.head_dim)


class DeviceCache:
    """A device's paged key-value cache, and the pages of the prefix groups it holds."""

    def __init__(self, layer: Layer, pages: int, page_size: int = 16):
        shape = (pages, layer.heads_kv, page_size, layer.head_dim)
        self.k = torch.empty(shape, dtype=layer.weight.dtype, device="cuda")
        self.v = torch.empty_like(self.k)
        self.page_size = page_size
        self.free = list(range(pages - 1, -1, -1))
        self.groups = {}  # Stage.key of a prefix -> its full pages

    def keep(self, instance: int, held):
        """Lets go of a workflow's groups that are not in `held`, what its plan's slots on this device name."""
        for key in [k for k in self.groups if k[0] == instance and k[2] not in held]:
            self.release(self.groups.pop(key))

    def take(self, n: int, using=()):
        """n free pages; the groups cached longest, but those in `using`, go where too few are free."""
        for key in [k for k in self.groups if k not in using]:
            if n <= len(self.free):
                break
            self.release(self.groups.pop(key))
        if n > len(self.free):
            raise RuntimeError("the cache has %d free pages, %d are needed" % (len(self.free), n))
        return [self.free.pop() for _ in range(n)]

    def release(self, pages):
        self.free.extend(pages)


@dataclasses.dataclass
class Stage:
    """A stage of a wave: its prefix group (0 = none), the tokens of the shared prefix, its own tokens, its model, the
    workflow that it is a stage of."""

    group: int
    prefix: torch.Tensor  # [P, hidden] token rows
    own: torch.Tensor     # [n, hidden], at least one
    model: int = 0
    instance: int = 0

    @property
    def key(self):
        """What a device caches a prefix as: its keys and values are a model's, and each workflow's plan has slots of its own."""
        return self.instance, self.model, self.group


def _ints(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


class Step:
    """The device arrays of one call over several sequences: new tokens of each, keys with them, pages."""

    def __init__(self, new, keys, pages):
        off = [0]
        for n in new:
            off.append(off[-1] + n)
        width = max(len(p) for p in pages)
        self.off, self.kv_len = _ints(off), _ints(keys)
        self.pages = _ints([p + [-1] * (width - len(p)) for p in pages])
        self.max_new = max(new)


def _store(layer, cache, step, x):
    """Project token rows, rotate queries and keys in place and store keys and values: the fused projection's queries and
    keys lie side by side, so one call rotates both (as query heads) while it stores.  Returns (q, k, v) views."""
    qkv, hq, hk = layer.project(x), layer.heads_q, layer.heads_q + layer.heads_kv
    k = qkv[:, hq:hk].clone()  # the call reads the keys as they come
    fate.fate_kv_append(qkv[:, :hk], k, qkv[:, hk:], cache.k, cache.v, step.off, step.kv_len, step.pages, layer.table,
                        q_out=qkv[:, :hk])
    return qkv[:, :hq], qkv[:, hq:hk], qkv[:, hk:]


def run_stages(layer: Layer, cache: DeviceCache, stages, answer_tokens: int = 0, reuse: bool = True):
    """Stages of one model, whose layer this is: attention outputs [n, heads_q, head_dim] of each stage's own tokens and of
    its answer tokens (list of [answer_tokens, heads_q, head_dim]), and how many prefix tokens were found in the cache.
    ``reuse`` False ignores the cached prefixes (and caches none)."""
    mine = []  # the pages taken for each stage
    try:
        return _run_stages(layer, cache, stages, answer_tokens, reuse, mine)
    finally:
        kept = {p for group in cache.groups.values() for p in group}
        cache.release([p for extra in mine for p in extra if p not in kept])


def _run_stages(layer, cache, stages, answer_tokens, reuse, mine):
    P, hq, d = cache.page_size, layer.heads_q, layer.head_dim
    pages, keys, cached, outs = [], [], [], [None] * len(stages)
    using = {s.key for s in stages}
    for s in stages:
        have = cache.groups.get(s.key, []) if reuse and s.group else []
        have = have[:s.prefix.shape[0] // P]
        total = s.prefix.shape[0] + s.own.shape[0]
        if total + answer_tokens > layer.table.shape[0]:
            raise ValueError("a stage of %d tokens with %d of an answer stands past the layer's %d positions" % (
                total, answer_tokens, layer.table.shape[0]))
        extra = cache.take(-(-(total + answer_tokens) // P) - len(have), using)
        mine.append(extra)
        pages.append(have + extra)
        keys.append(total)
        cached.append(len(have) * P)
    for hit in (False, True):
        of = [i for i in range(len(stages)) if (cached[i] > 0) == hit]
        if not of:
            continue
        # what is not in the cache: the prefix's last tokens (those short of a full page, or all) and the stage's own
        rows = [torch.cat([stages[i].prefix[cached[i]:], stages[i].own]) for i in of]
        step = Step([r.shape[0] for r in rows], [keys[i] for i in of], [pages[i] for i in of])
        q, k, v = _store(layer, cache, step, torch.cat(rows))
        if hit:
            out, _ = fate.fate_attn_paged(q, cache.k, cache.v, step.off, step.kv_len, step.pages, max_new=step.max_new)
        else:
            out, _ = fate.fate_attn_prompt(q, k, v, step.off)
        at = 0
        for i, r in zip(of, rows):
            at += r.shape[0]
            outs[i] = out[at - stages[i].own.shape[0]:at]
    answers = torch.empty((answer_tokens, len(stages), hq, d), dtype=layer.weight.dtype, device="cuda")
    if answer_tokens:
        step = Step([1] * len(stages), keys, pages)
        for t in range(answer_tokens):
            step.kv_len += 1
            # a model would feed the token it sampled; the layer's own output stands in for its embedding
            x = (answers[t - 1] if t else torch.stack([o[-1] for o in outs])).flatten(1)[:, :layer.weight.shape[0]]
            q, _, _ = _store(layer, cache, step, x.contiguous())
            fate.fate_attn_paged(q, cache.k, cache.v, step.off, step.kv_len, step.pages, max_new=1, out=answers[t])
    for s, p, n in zip(stages, pages, cached):
        full = p[:s.prefix.shape[0] // P]
        if reuse and s.group and n == 0 and full and s.key not in cache.groups:
            cache.groups[s.key] = full
    return outs, list(answers.unbind(1)), sum(cached)


class Prompts:
    """Random token rows for stages: a prefix per group (its length from the workload), own tokens per stage."""

    def __init__(self, w, hidden, dtype, own_tokens=(16, 256), seed=0):
        self.w, self.hidden, self.dtype, self.own = w, hidden, dtype, own_tokens
        self.gen = torch.Generator(device="cuda").manual_seed(seed)
        self.prefixes = {}

    def rows(self, n):
        return torch.randn(n, self.hidden, generator=self.gen, device="cuda").to(self.dtype)

    def stage(self, flat: int) -> Stage:
        group = int(self.w.prefix_hash[flat])
        if group not in self.prefixes:
            self.prefixes[group] = self.rows(int(self.w.prefix_tokens[flat]) if group else 0)
        lo, hi = self.own
        n = int(torch.randint(lo, hi + 1, (1,), generator=self.gen, device="cuda"))
        instance = int(np.searchsorted(self.w.stage_off, flat, side="right")) - 1
        return Stage(group, self.prefixes[group], self.rows(n), int(self.w.model[flat]), instance)


def follow_plan(w, waves: int, k: int = 4):
    """Waves of a plan, one after the other: (flat stage id, device) of the single-device placements (a window's shards are
    left out), and the prefix groups that the plan's slots hold on each device as the wave starts, [instances, devices, slots]."""
    packed = fate.fate_pack_dags(w)
    state = fate.fate_pack_state(packed, w, advance=True)
    params = fate.make_params(w)
    for _ in range(waves):
        F = state.counts()[0]
        if F == 0:
            return
        _, idx, val = fate.fate_score_topk(packed, state, params, k)
        sel = fate.fate_plan_wave(state, idx, val)
        flat = fate.frontier_table(state)[0]
        chosen = sel[:F].cpu().tolist()
        yield [(int(flat[f]), c) for f, c in enumerate(chosen) if 0 <= c < w.D], fate.state_arrays(state)["prefix_cache"]
        fate.fate_commit_advance(packed, state, sel)


def plan_waves(w, waves: int, k: int = 4):
    """The placements of :func:`follow_plan`."""
    for placed, _ in follow_plan(w, waves, k):
        yield placed


def carry_out(layers, caches, stages, devices, slots, answer_tokens: int = 0, reuse: bool = True):
    """A wave's stages, each on its device: what the plan's slots no longer name leaves the device's cache, then each model's
    stages go through its layer.  Returns how many prefix tokens were found cached."""
    found = 0
    for d, cache in enumerate(caches):
        for instance, held in enumerate(slots[:, d].tolist()):
            cache.keep(instance, held)
        here = [s for s, on in zip(stages, devices) if on == d]
        for model in sorted({s.model for s in here}):
            found += run_stages(layers[model], cache, [s for s in here if s.model == model], answer_tokens, reuse)[2]
    return found


def main(instances: int = 4, waves: int = 12, answer_tokens: int = 4):
    """Plan waves and carry out every device's share here, one device after the other, each with a cache of its own."""
    w = synth.make_workload("forkjoin-4096x1000-d16", B=instances)
    layers = [Layer.random(seed=m) for m in range(w.M)]
    caches = [DeviceCache(layers[0], pages=1 << 13) for _ in range(w.D)]
    prompts = Prompts(w, layers[0].weight.shape[0], layers[0].weight.dtype)
    run_stages(layers[0], caches[0], [Stage(0, prompts.rows(0), prompts.rows(8))], 1)  # libraries load at the first call
    for number, (placed, slots) in enumerate(follow_plan(w, waves)):
        stages, devices = [prompts.stage(flat) for flat, _ in placed], [d for _, d in placed]
        took, found = {}, 0
        for reuse in (False, True) if number % 2 else (True, False):  # neither is always the first to meet the wave's shapes
            torch.cuda.synchronize()
            t = time.perf_counter()
            found = max(found, carry_out(layers, caches, stages, devices, slots, answer_tokens, reuse))
            torch.cuda.synchronize()
            took[reuse] = (time.perf_counter() - t) * 1e3
        tokens = sum(s.prefix.shape[0] + s.own.shape[0] for s in stages)
        print("wave %d: %d stages on %d devices, %d prompt tokens, %d of them cached: %.2f ms, %.2f without the cached ones"
              % (number, len(stages), len(set(devices)), tokens, found, took[True], took[False]), flush=True)


if __name__ == "__main__":
    main()

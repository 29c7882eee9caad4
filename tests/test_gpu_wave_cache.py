"""The wave example's page cache: what it holds, gives back and refuses."""

import pytest
import torch

from paper_2605_07238_amd import synth, wave

pytestmark = pytest.mark.gpu


def layer(positions=512, seed=3):
    return wave.Layer.random(hidden=64, heads_q=4, heads_kv=2, head_dim=64, positions=positions, dtype=torch.float16, seed=seed)


def rows(n, seed=0):
    return torch.randn(n, 64, generator=torch.Generator(device="cuda").manual_seed(seed), device="cuda").half()


def test_a_wave_that_does_not_fit_takes_no_pages():
    one = layer()
    cache = wave.DeviceCache(one, pages=12)
    fits, more = wave.Stage(1, rows(64), rows(20)), wave.Stage(2, rows(64), rows(40))  # 6 and 7 pages
    with pytest.raises(RuntimeError):
        wave.run_stages(one, cache, [fits, more])
    assert sorted(cache.free) == list(range(12)) and not cache.groups
    outs, _, found = wave.run_stages(one, cache, [fits])
    assert found == 0 and outs[0].shape == (20, 4, 64) and len(cache.free) == 8


@pytest.mark.parametrize("prefix,own,answers", [(0, 513, 0), (500, 13, 0), (480, 20, 13)])
def test_positions_past_the_rotation_table_are_refused(prefix, own, answers):
    one = layer(positions=512)
    cache = wave.DeviceCache(one, pages=64)
    with pytest.raises(ValueError, match="positions"):
        wave.run_stages(one, cache, [wave.Stage(1, rows(prefix), rows(own))], answers)
    assert len(cache.free) == 64
    wave.run_stages(one, cache, [wave.Stage(1, rows(prefix), rows(512 - prefix - answers))], answers)


def test_models_do_not_share_keys():
    """A prefix group that stages of two models start with: each model's keys and values serve its own stages alone."""
    a, b = layer(seed=3), layer(seed=4)
    cache = wave.DeviceCache(a, pages=64)
    prefix, own = rows(48, 1), rows(20, 2)
    first = wave.run_stages(a, cache, [wave.Stage(7, prefix, own, model=0)])
    other = wave.run_stages(b, cache, [wave.Stage(7, prefix, own, model=1)])
    assert first[2] == other[2] == 0
    fresh = wave.run_stages(b, wave.DeviceCache(b, pages=64), [wave.Stage(7, prefix, own, model=1)])
    assert torch.equal(other[0][0], fresh[0][0])
    assert wave.run_stages(a, cache, [wave.Stage(7, prefix, own, model=0)])[2] == 48
    assert wave.run_stages(b, cache, [wave.Stage(7, prefix, own, model=1)])[2] == 48


def test_the_cache_holds_what_the_plan_says():
    """Groups that the plan's slots no longer name are let go, for their workflow alone."""
    one = layer()
    cache = wave.DeviceCache(one, pages=64)
    stages = [wave.Stage(g, rows(32, g), rows(5, 50 + g), instance=b) for b, g in ((0, 7), (0, 8), (1, 7), (1, 9))]
    assert wave.run_stages(one, cache, stages)[2] == 0 and len(cache.free) == 56
    cache.keep(0, [8, 0, 0])
    assert len(cache.free) == 58
    assert [wave.run_stages(one, cache, [s], reuse=True)[2] for s in stages[1:]] == [32, 32, 32]
    cache.keep(0, [])
    cache.keep(1, [9])
    assert len(cache.free) == 62
    assert [wave.run_stages(one, cache, [s])[2] for s in (stages[3], stages[2], stages[2])] == [32, 0, 32]


def test_a_full_cache_lets_its_oldest_groups_go():
    one = layer()
    cache = wave.DeviceCache(one, pages=12)
    stages = [wave.Stage(g, rows(48, g), rows(10, 50 + g)) for g in range(1, 9)]  # three full pages and one more
    for s in stages:
        assert wave.run_stages(one, cache, [s])[2] == 0
    assert len(cache.groups) == 3 and len(cache.free) == 3
    assert [wave.run_stages(one, cache, [s])[2] for s in (stages[7], stages[6], stages[5], stages[0])] == [48, 48, 48, 0]
    # not those that the same call reads
    out, _, found = wave.run_stages(one, cache, [stages[0], stages[7], stages[4]])
    assert found == 96
    fresh = wave.DeviceCache(one, pages=64)
    for s, got in zip((stages[0], stages[7], stages[4]), out):
        want = wave.run_stages(one, fresh, [s])[0][0]
        assert torch.allclose(got.float(), want.float(), atol=0.02, rtol=0.02)


def test_waves_follow_the_slots_of_the_plan():
    """Over the waves of a plan, a device's cache never holds a group that the plan's slots there do not name."""
    w = synth.make_workload("forkjoin-4096x1000-d16", B=3)
    layers = [wave.Layer.random(hidden=64, heads_q=2, heads_kv=1, head_dim=64, seed=m) for m in range(w.M)]
    caches = [wave.DeviceCache(layers[0], pages=1 << 12) for _ in range(w.D)]
    prompts = wave.Prompts(w, 64, layers[0].weight.dtype, own_tokens=(1, 20))
    hits = let_go = 0
    for placed, slots in wave.follow_plan(w, 30):
        before = [set(c.groups) for c in caches]
        hits += wave.carry_out(layers, caches, [prompts.stage(f) for f, _ in placed], [d for _, d in placed], slots)
        for d, cache in enumerate(caches):
            held = {(b, int(g)) for b in range(w.B) for g in slots[b, d]}
            here = {(prompts.stage(f).instance, int(w.prefix_hash[f])) for f, on in placed if on == d}
            assert all((b, g) in held | here for b, _, g in cache.groups)
            let_go += len(before[d] - set(cache.groups))
    assert hits > 0 and let_go > 0

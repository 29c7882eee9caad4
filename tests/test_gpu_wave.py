"""The wave example: a stage whose prefix is cached gets what it gets when its whole prompt is attended."""

import numpy as np
import pytest
import torch

import attn_oracle as ao
from paper_2605_07238_amd import synth, wave

pytestmark = pytest.mark.gpu


def small_layer():
    return wave.Layer.random(hidden=64, heads_q=4, heads_kv=2, head_dim=64, positions=512, dtype=torch.float16, seed=3)


def whole(layer, stage):
    """The stage's own rows from the definition, in 64 bits, and their bound; projections as the layer has them."""
    x = torch.cat([stage.prefix, stage.own])
    qkv = layer.project(x).double().cpu().numpy()
    table = layer.table.double().cpu().numpy()
    n = x.shape[0]
    rot, _ = ao.rotate(qkv[:, :6], np.arange(n), table, False)
    rot = torch.from_numpy(rot).half().double().numpy()  # rounded once, as stored
    return ao.attend(rot[:, :4], rot[:, 4:6], qkv[:, 6:], 1 + np.arange(n), 0.125)


@pytest.mark.parametrize("prefix", [0, 5, 16, 37, 160])
def test_cached_prefix_gives_the_same_rows(prefix):
    layer = small_layer()
    cache = wave.DeviceCache(layer, pages=64)
    gen = torch.Generator(device="cuda").manual_seed(prefix)
    rows = lambda n: torch.randn(n, 64, generator=gen, device="cuda").half()  # noqa: E731
    shared = rows(prefix)
    first, second = wave.Stage(7, shared, rows(21)), wave.Stage(7, shared, rows(40))
    other = wave.Stage(0, rows(0), rows(3))
    pages = len(cache.free)
    out1, ans1, found = wave.run_stages(layer, cache, [first, other], 3)
    assert found == 0 and len(ans1) == 2 and ans1[0].shape == (3, 4, 64)
    out2, ans2, found = wave.run_stages(layer, cache, [second, other], 3)
    assert found == prefix // 16 * 16
    again, ans3, found = wave.run_stages(layer, cache, [second, other], 3, reuse=False)
    assert found == 0 and len(cache.free) == pages - prefix // 16
    for stage, got in ((first, out1[0]), (second, out2[0]), (second, again[0]), (other, out2[1])):
        out, _, tol, _ = whole(layer, stage)
        n = stage.own.shape[0]
        # rotated queries and keys may round the other way where float32 and float64 differ: one more rounding of each score
        bound = tol[-n:] + 4 * ao.UNIT[torch.float16] * (np.abs(out[-n:]) + 1)
        assert (np.abs(got.double().cpu().numpy() - out[-n:]) <= bound).all()
    # answers: the cached and the whole route see the same keys up to their roundings
    for a, b in zip(ans2, ans3):
        assert torch.allclose(a.float(), b.float(), atol=0.05, rtol=0.05)


def test_a_planned_wave_runs(capsys):
    w = synth.make_workload("forkjoin-4096x1000-d16", B=2)
    waves = list(wave.plan_waves(w, 2))
    assert waves and all(0 <= d < w.D for x in waves for _, d in x)
    assert len({(f, d) for x in waves for f, d in x}) == sum(map(len, waves))
    wave.main(instances=2, waves=3, answer_tokens=2)
    assert "prompt tokens" in capsys.readouterr().out

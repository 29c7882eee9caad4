"""fate_sample against its definition, row by row: the same tokens, and the logarithms of their shares."""

import numpy as np
import pytest
import torch

import serve_oracle as so
from paper_2605_07238_amd import fate

pytestmark = pytest.mark.gpu
BF, HF, FF = torch.bfloat16, torch.float16, torch.float32
LAST = float(np.nextafter(np.float32(1), np.float32(0)))
DEFAULTS = dict(temperature=1.0, top_k=0, top_p=1.0, min_p=0.0)


def check(logits, u, layout=None, **settings):
    """logits [R, V] on the CPU, settings as numbers or lists by row."""
    R = logits.shape[0]
    x = logits.cuda() if layout is None else layout(logits)
    given = {}
    for name, value in settings.items():
        kind = torch.int32 if name == "top_k" else torch.float32
        given[name] = torch.tensor(value, dtype=kind).cuda() if isinstance(value, list) else value
    status = torch.zeros(R, dtype=torch.int32, device="cuda")
    du = torch.tensor(u, dtype=torch.float32).cuda()
    token, logprob = fate.fate_sample(x, du, logprob=True, status=status, **given)
    only, none = fate.fate_sample(x, du, **given)
    assert none is None and torch.equal(only, token) and not status.any()
    rows = logits.double().numpy()
    for r in range(R):
        own = {k: (v[r] if isinstance(v, list) else v) for k, v in dict(DEFAULTS, **settings).items()}
        own = {k: float(np.float32(v)) if k != "top_k" else v for k, v in own.items()}
        want, share = so.sample(rows[r], u=float(np.float32(u[r])), **own)
        assert token[r].item() == want, (r, own, u[r])
        got = logprob[r].item()
        # the result's rounding; a share's sum and weight are off by some 2^-40
        assert got == share or abs(got - share) <= 2.0 ** -23 * abs(share) + 2.0 ** -38
    return token


def logits_of(R, V, dtype, seed, spread=2.5):
    gen = torch.Generator().manual_seed(seed)
    x = torch.randn(R, V, generator=gen) * spread
    some = torch.randint(0, V, (R, min(V, 20)), generator=gen)
    return x.scatter_(1, some, torch.randn(R, some.shape[1], generator=gen) * 2 + 8).to(dtype)


def uniform(R, seed):
    return torch.rand(R, generator=torch.Generator().manual_seed(seed + 1000)).tolist()


FILTERS = [dict(), dict(top_k=1), dict(top_k=40), dict(top_p=0.9), dict(min_p=0.05), dict(top_k=50, top_p=0.8),
           dict(top_k=200, top_p=0.95, min_p=0.02), dict(top_k=3000), dict(top_k=5000, top_p=0.97), dict(top_p=0.99, min_p=0.001),
           dict(top_k=2000, min_p=0.3), dict(top_p=0.01), dict(min_p=1.0), dict(top_k=1024), dict(top_k=1025, top_p=0.999)]
SIZES = [1, 2, 7, 64, 65, 1000, 4095, 4096, 4097, 5003, 32000, 50001, 131072, 200003]


@pytest.mark.parametrize("filters", FILTERS, ids=str)
@pytest.mark.parametrize("V", SIZES)
def test_sizes(V, filters):
    which = SIZES.index(V) + FILTERS.index(filters)
    dtype = [FF, BF, HF][which % 3]
    check(logits_of(5, V, dtype, which), [0.0, LAST] + uniform(3, which), temperature=[1.0, 0.7, 1.3, 0.2, 2.0], **filters)


@pytest.mark.parametrize("dtype", [FF, BF, HF], ids=["f32", "bf16", "f16"])
@pytest.mark.parametrize("V", [900, 20000])
def test_rows_with_settings_of_their_own(V, dtype):
    R, rng = 120, np.random.default_rng(V)
    check(logits_of(R, V, dtype, V), uniform(R, V), temperature=rng.choice([0.0, 0.3, 0.8, 1.0, 1.7], R).tolist(),
          top_k=rng.choice([0, 1, 2, 30, 1000, 1500, V, V + 5], R).tolist(), top_p=rng.choice([1.0, 0.9, 0.5, 0.999], R).tolist(),
          min_p=rng.choice([0.0, 0.0, 0.01, 0.5], R).tolist())


@pytest.mark.parametrize("V", [6, 4096, 4100, 70000])
@pytest.mark.parametrize("values", [1, 2, 5])
def test_equal_logits(V, values):
    """Few distinct values: ties go to the lowest indices, whatever holds the cut."""
    gen = torch.Generator().manual_seed(V + values)
    x = torch.randint(0, values, (8, V), generator=gen).float() * 0.5
    u = [0.0, LAST, 0.5, 0.25] + uniform(4, V)
    for filters in (dict(), dict(top_k=3), dict(top_k=V // 2), dict(top_k=1500), dict(top_p=0.5), dict(top_p=0.3, top_k=V - 1),
                    dict(min_p=0.7), dict(top_k=V // 3 + 1, top_p=0.75), dict(top_k=1024, top_p=0.25)):
        check(x, u, **filters)


def test_borders():
    """Sums that are whole numbers: u and top_p right at a border."""
    for V, dtype in ((8, FF), (1 << 13, BF), (1 << 17, HF)):
        x = torch.full((9, V), 1.5).to(dtype)
        u = [0.0, 0.125, 0.25, 0.375, 0.5, 0.625, 0.75, 0.875, LAST]
        token = check(x, u)
        assert token.tolist()[:8] == [V // 8 * i for i in range(8)] and token[8] == V - 1
        token = check(x, u, top_p=0.5)
        assert token.tolist()[:8] == [V * i // 16 for i in range(8)] and token[8] == V // 2 - 1
        token = check(x, u, top_k=4, top_p=0.75)
        assert token.tolist() == [0, 0, 0, 1, 1, 1, 2, 2, 2]


def test_no_token_and_infinities():
    inf, nan = float("inf"), float("nan")
    for V in (5, 9000):
        x = torch.full((9, V), -inf)
        x[1] = nan
        x[2, V - 2] = -3e38
        x[3, 1], x[3, 3] = inf, inf
        x[4, 2], x[4, 4] = nan, 0.0
        x[5, 0], x[5, 3] = 3e38, -3e38
        x[6, :3] = torch.tensor([1e-45, 0.0, -1e-45])
        x[7, 1], x[7, 4] = -0.0, 0.0
        x[8, 2], x[8, 3], x[8, 4] = inf, nan, 1.0
        for filters in (dict(), dict(top_k=2), dict(top_p=0.6), dict(min_p=0.1), dict(temperature=0.0), dict(top_k=1), dict(top_k=3000),
                        dict(temperature=1e-30), dict(temperature=1e-45), dict(temperature=3e38)):
            token = check(x, [0.6] * 9, **filters).tolist()
            assert token[:3] == [-1, -1, V - 2] and token[4] == 4
    check(torch.full((2, 6), 65504.0).half() * torch.tensor([1.0, -1.0])[:, None].half(), [0.3, 0.9], top_p=0.5)


def test_layouts():
    """Odd strides and places, one element at a time and one row for all."""
    for dtype in (FF, BF, HF):
        for V in (33, 6001):
            x, u = logits_of(7, V, dtype, V), uniform(7, V)

            def shifted(t, by, gap):
                wide = torch.full((7 * (V + gap) + by,), float("inf"), dtype=dtype, device="cuda")
                view = wide[by:].as_strided((7, V), (V + gap, 1), by)
                return view.copy_(t)

            for by, gap in ((1, 0), (3, 1), (5, 7), (8, 8), (7, 2)):
                for filters in (dict(), dict(top_k=20), dict(top_p=0.9)):
                    check(x, u, lambda t: shifted(t, by, gap), **filters)
            check(x[:1].expand(7, V), u, lambda t: t[:1].cuda().expand(7, V), top_p=0.9)
    assert fate.fate_sample(torch.empty(0, 9, device="cuda"), torch.empty(0, device="cuda"))[0].shape == (0,)


def few_values(kind, R, V, dtype, seed):
    gen = torch.Generator().manual_seed(seed)
    x = torch.randn(R, V, generator=gen)
    if kind == "wide":  # more values than a table of weights holds, on both sides of zero
        x = torch.sign(x) * torch.exp2(torch.rand(R, V, generator=gen) * (60 if dtype == BF else 20) - (50 if dtype == BF else 12))
    elif kind == "zeros":
        x = torch.where(x.abs() < 1.2, torch.copysign(torch.zeros(()), torch.randn(R, V, generator=gen)), x)
    elif kind == "tiny":
        x *= 1e-30 if dtype == BF else 1e-6
    elif kind == "below zero":
        x = x * 2 - 60
    elif kind == "holes":
        x[torch.rand(R, V, generator=gen) < 0.3] = -float("inf")
        x[torch.rand(R, V, generator=gen) < 0.3] = float("nan")
    elif kind == "infinite":
        x[::2, ::max(1, V // 3)] = float("inf")
        x[1, :] = -float("inf")
    elif kind == "crowded":  # one value more often than 16 bits count
        x[:, :V - V // 8] = 0.75
    return x.to(dtype)


@pytest.mark.parametrize("kind", ["plain", "wide", "zeros", "tiny", "below zero", "holes", "infinite", "crowded"])
@pytest.mark.parametrize("V", [8192, 16384, 16391, 100003, 131072])
@pytest.mark.parametrize("dtype", [BF, HF], ids=["bf16", "f16"])
def test_few_values(dtype, V, kind):
    """Cuts among the values of 16-bit logits, in calls of one setting and, of long rows too, of a setting for each row."""
    seed = V + len(kind)
    x, u = few_values(kind, 6, V, dtype, seed), [0.0, LAST] + uniform(4, seed)
    for filters in (dict(top_p=0.9), dict(top_k=257), dict(top_k=V - 1, top_p=0.5), dict(top_k=V // 3, min_p=0.9), dict(top_p=0.97, min_p=0.02),
                    dict(top_p=0.999, temperature=50.0), dict(top_p=0.5, temperature=1e-4), dict(top_p=1e-6), dict(top_k=V // 2, temperature=1e30)):
        check(x, u, **filters)
    check(x, u, temperature=[1.0, 0.5, 0.0, 3.0, 1.0, 9.0], top_k=[0, 3000, 5, 0, V - 5, 0], top_p=[0.9, 0.8, 0.7, 1.0, 1.0, 0.999],
          min_p=[0.0, 0.0, 0.1, 0.0, 0.2, 0.0])


def test_more_rows_than_the_chip_runs():
    R = 3001
    check(logits_of(R, 70, FF, 0), uniform(R, 0), top_p=0.9)


def test_settings_out_of_range():
    nan, inf = float("nan"), float("inf")
    bad = dict(temperature=[-1.0, nan, inf, -0.0], top_k=[-1, -(1 << 31)], top_p=[0.0, -0.5, 1.5, nan], min_p=[-0.1, 1.1, nan],
               u=[-0.1, 1.0, nan, inf])
    for V in (50, 9000):
        x = logits_of(6, V, FF, V).cuda()
        for name, values in bad.items():
            for value in values:
                kind = torch.int32 if name == "top_k" else torch.float32
                row = dict(u=0.5, **DEFAULTS)[name]
                settings = {name: torch.tensor([row] * 2 + [value] + [row] * 3, dtype=kind).cuda()}
                u = settings.pop("u", torch.full((6,), 0.5, device="cuda"))
                status = torch.zeros(6, dtype=torch.int32, device="cuda")
                token, logprob = fate.fate_sample(x, u, logprob=True, status=status, **settings)
                clean, _ = fate.fate_sample(x, torch.full((6,), 0.5, device="cuda"))
                wrong = not (name == "temperature" and value == 0)
                assert status.tolist() == [0, 0, -1 if wrong else 0, 0, 0, 0]
                keep = [0, 1, 3, 4, 5]
                assert token[keep].tolist() == clean[keep].tolist()
                assert not wrong or (token[2] == -1 and logprob[2] == -inf)


def test_captured_and_on_another_stream():
    x = logits_of(40, 9001, BF, 3).cuda()
    u, p, out = torch.rand(40, device="cuda"), torch.full((40,), 0.9, device="cuda"), torch.empty(40, dtype=torch.int32, device="cuda")
    ws = torch.empty(fate.fate_sample_ws_size(x), dtype=torch.uint8, device="cuda")
    go = lambda **m: fate.fate_sample(x, u, 0.8, top_p=p, **m)[0]  # noqa: E731
    go(out=out, ws=ws)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    other = go(stream=side)
    side.synchronize()
    assert torch.equal(out, other)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        go(out=out, ws=ws)
    for step in range(5):
        u.copy_(torch.rand(40))
        p -= 0.1
        x += torch.randn_like(x)
        graph.replay()
        assert torch.equal(go(), out)


def test_what_the_binding_refuses():
    x, u = logits_of(4, 50, FF, 0).cuda(), torch.rand(4, device="cuda")
    ones, ints = torch.ones(4, device="cuda"), torch.ones(4, dtype=torch.int32, device="cuda")
    assert fate.fate_sample(x, u, ones, ints, ones, ones)[0].shape == (4,)
    for args in ((x[0], u), (x.double(), u), (x.t(), u), (x.int(), u), (x, u[:3]), (x, u.double()), (x, u.cpu()), (x, u, ones.double()),
                 (x, u, ones, ones), (x, u, ones, ints.long()), (x, u, ones, ints, ones[:2]), (x, u, ones, ints, ones, ints)):
        with pytest.raises(ValueError):
            fate.fate_sample(*args)
    for bad in (dict(temperature=-1.0), dict(temperature=float("inf")), dict(top_k=-1), dict(top_p=0.0), dict(top_p=1.1), dict(min_p=-0.1),
                dict(min_p=1.5), dict(top_p=float("nan"))):
        with pytest.raises(fate.FateError):
            fate.fate_sample(x, u, **bad)
    with pytest.raises(fate.FateError):
        fate.fate_sample(x[:, :0], u)
    with pytest.raises(ValueError, match="gradient"):
        fate.fate_sample(x.clone().requires_grad_(), u)
    with torch.no_grad():
        fate.fate_sample(x.clone().requires_grad_(), u)


@pytest.mark.parametrize("R,V", [(3, 5003), (3, 131072), (130, 131072), (2, 1 << 20)], ids=str)
@pytest.mark.parametrize("top_p", [1e-7, 1e-14, 1e-30, 1e-45])
def test_top_p_below_what_bins_hold(top_p, R, V):
    """A top_p of less than the units of the bins' sums keeps the largest logit alone (the next one has a weight of 1 before
    it, the aim is below V times 1e-7), whatever min_p leaves: thousands of flat logits here."""
    x = torch.rand(2, V, generator=torch.Generator().manual_seed(V))
    x[0, V // 3] = x[0, V - 2] = x[1, 5] = 1.25
    rows = x[torch.arange(R) % 2].cuda()
    u = torch.linspace(0, LAST, R).cuda()
    want = torch.tensor([V // 3, 5], dtype=torch.int32)[torch.arange(R) % 2]
    for filters in (dict(min_p=0.01), dict(min_p=0.9), dict(), dict(top_k=1000, min_p=0.01), dict(top_k=V - 1, min_p=0.01)):
        for temperature in (1.0, 1.5):
            token, logprob = fate.fate_sample(rows, u, temperature, top_p=top_p, logprob=True, **filters)
            assert torch.equal(token.cpu(), want) and not logprob.any(), (filters, temperature)
    check(x, [0.3, LAST], top_p=top_p, min_p=0.01)


def tail(V):
    """One large logit, and V - 1 of weights that the bins of a row of 2^20 round to nothing."""
    x = -29.25 + 0.1 * torch.rand(1, V, generator=torch.Generator().manual_seed(V))
    x[0, V // 2] = 0.0
    return x


@pytest.mark.parametrize("R", [2, 129])
def test_top_p_in_a_tail_that_bins_do_not_hold(R):
    """The cut of top_p lies among tokens whose weights together are 2e-7 of the whole: sums of whole numbers do not reach it.
    A smaller min_p must not stand in for it."""
    V, us, settings = 1 << 20, [LAST, 1 - 2.0 ** -23, 0.5, 0.0], dict(top_p=LAST, min_p=float(np.float32(1e-30)))
    x = tail(V)
    row = x.double().numpy()[0]
    w = np.exp(row.astype(np.longdouble))
    order = np.argsort(-row, kind="stable")
    before = w[order].cumsum() - w[order]
    kept = before < np.longdouble(LAST) * w.sum()
    assert V // 2 < kept.sum() < 0.9 * V
    upto = np.where(np.isin(np.arange(V), order[kept]), w, 0).cumsum()
    dx = x.cuda().expand(R, V)
    for u in us:
        # float64 sums and the cut may be off by some 2e-15, a hundredth of a token: u is not that near a border
        t = np.longdouble(u) * upto[-1]
        want, share = so.sample(row, u=u, **settings)
        assert upto[want] - t > 2e-14 and t - (upto[want] - w[want]) > 2e-14 or u == 0
        token, logprob = fate.fate_sample(dx, torch.full((R,), u, device="cuda"), logprob=True, **settings)
        assert (token == want).all() and (logprob - share).abs().max() <= 2.0 ** -23 * abs(share) + 2.0 ** -38, u


def test_top_k_past_32_bits_cuts_nothing():
    x, u = logits_of(4, 300, FF, 1).cuda(), torch.tensor(uniform(4, 2)).cuda()
    want = fate.fate_sample(x, u)[0]
    for k in ((1 << 31) - 1, 1 << 31, (1 << 32) + 1, (1 << 63) - 1, 1 << 70):
        assert torch.equal(fate.fate_sample(x, u, top_k=k)[0], want), k
    for k in (-1, -(1 << 31) - 1, -(1 << 32) + 1, -(1 << 70)):
        with pytest.raises(fate.FateError):
            fate.fate_sample(x, u, top_k=k)
    with pytest.raises(TypeError):
        fate.fate_sample(x, u, top_k=2.0)

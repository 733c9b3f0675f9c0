"""Tokens drawn on the GPU against oracle/operators.py: types, vocabularies, rules, ties,
masks, extreme choices, strides, the same draws again and from a graph.

A drawn token hangs on comparisons of sums in 64 bits. The oracle says how near, relative
to the sum, the nearest of a row's comparisons came (`margin`); sums of V weights, each
within 2^-46 of its size or better, are within V 2^-46 of the sum in any order, so a row
whose margin is above that has one right token. Rows below it may not have another token
than one that the comparisons' other side gives: there are none in these cases, which is
asserted, but where the sums are exact (equal logits). logp: the quotient of two such sums'
logarithm, rounded to 32 bits."""
import numpy as np
import pytest

from oracle import operators as OO
from tests.gpu_common import announce, device
from tests.test_gpu_operators import _dtype, _put

pytestmark = pytest.mark.gpu


def _call(logits, u, temperature=None, top_k=None, top_p=None, min_p=None, wide=False):
    import torch
    from paper_2606_06742_amd import kmpath as km
    T, V = logits.shape
    f = lambda a: None if a is None else torch.as_tensor(np.asarray(a, np.float32), device=device())
    k = None if top_k is None else torch.as_tensor(np.asarray(top_k, np.int32), device=device())
    tokens = torch.full((T,), -7, dtype=torch.int64 if wide else torch.int32, device=device())
    logp = torch.full((T,), 7.0, device=device())
    ws = torch.full((km.kmp_sample_tokens_workspace_bytes(T, V),), 255, dtype=torch.uint8, device=device())
    km.kmp_sample_tokens(logits, f(u), tokens, f(temperature), k, f(top_p), f(min_p), logp, ws)
    return tokens.cpu().numpy(), logp.double().cpu().numpy()


def _check(logits, values, u, exact=False, **rules):
    f = lambda a: None if a is None else np.asarray(a, np.float32).astype(np.float64)
    r = {k: (v if k == "top_k" else f(v)) for k, v in rules.items()}
    te, le, margin = OO.sample_tokens(values, f(u), **r)
    tokens, logp = _call(logits, u, **rules)
    V = values.shape[1]
    assert exact or np.all(margin > V * 2.0 ** -46), margin.min()
    assert np.array_equal(tokens, te), (np.flatnonzero(tokens != te), tokens, te)
    assert np.array_equal(np.isnan(logp), np.isnan(le)) and np.array_equal(logp == -np.inf, le == -np.inf)
    fine = np.isfinite(le)
    assert np.all(np.abs(logp[fine] - le[fine]) <= 2.0 ** -24 * np.abs(le[fine]) + V * 2.0 ** -45)
    return tokens


def _logits(rng, T, V, spread=2.0):
    x = spread * rng.standard_normal((T, V))
    x[:, rng.integers(0, V, 5)] += 6.0
    return x


RULES = [dict(), dict(top_k=1), dict(top_k=7), dict(top_k=300), dict(top_k=1500), dict(top_p=0.9), dict(top_p=0.3),
         dict(top_p=0.999), dict(min_p=0.05), dict(min_p=1e-4), dict(top_k=50, top_p=0.8), dict(top_k=2000, top_p=0.95),
         dict(top_p=0.95, min_p=0.01), dict(top_k=40, top_p=0.9, min_p=0.02), dict(top_k=3000, min_p=1e-3)]


@pytest.mark.parametrize("xt", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("V,pad,off", [(1, 0, 0), (2, 0, 0), (7, 1, 1), (64, 0, 0), (1000, 0, 0), (1023, 3, 1), (1025, 0, 0),
                                       (4099, 1, 0), (32000, 0, 0), (50257, 0, 1), (128000, 0, 0)])
def test_rules(xt, V, pad, off):
    """Every rule at every length, each row with choices of its own."""
    T = 6 if V < 20000 else 3
    rng = np.random.default_rng(V + pad)
    logits, values = _put(_logits(rng, T, V), _dtype(xt), pad, off)
    for rule in RULES:
        announce(f"sample {xt} {T} x {V} gap {pad} offset {off} {rule}")
        u = rng.random(T)
        r = {k: np.full(T, v) * (rng.uniform(0.9, 1.0, T) if k != "top_k" else 1) for k, v in rule.items()}
        if "top_k" in r:
            r["top_k"] = r["top_k"].astype(np.int32)
        for temperature in (None, 0.5 + rng.random(T)):
            _check(logits, values, u, temperature=temperature, **r)


def test_choices_of_their_own():
    """Rows of one call with different choices, the extremes among them: greedy, one
    token, all tokens, everything but the best ruled out, u of 0 and of 1."""
    rng = np.random.default_rng(3)
    T, V = 16, 5001
    logits, values = _put(_logits(rng, T, V), _dtype("f32"), 2, 1)
    inf = np.inf
    temperature = np.array([0.0, -1.0, 1.0, 1.0, 1e-3, 100.0, 1.0, 1.0, 0.7, 1.0, 1.0, 1.0, 1e-30, 0.3, 1.0, 1.0])
    top_k = np.array([0, 5, 1, -3, 0, 0, V, V + 10, 2 ** 31 - 1, 0, 0, 0, 0, V - 1, 2, 0], np.int32)
    top_p = np.array([1.0, 0.5, 0.5, 1.5, inf, 0.9, 0.0, -1.0, 1e-20, 1.0, 0.9999, 1.0, 0.5, 1.0, 0.99, 1.0])
    min_p = np.array([0.0, 0.0, 0.0, -1.0, 0.0, 0.0, 0.0, 0.0, 0.0, 1.0, 2.0, 0.0, 0.0, 0.0, 0.0, 1e-30])
    u = rng.random(T)
    u[3], u[11], u[15] = 0.0, 1.0, -0.5
    announce("sample, choices of their own")
    tokens = _check(logits, values, u, temperature=temperature, top_k=top_k, top_p=top_p, min_p=min_p, exact=True)
    best = values.argmax(axis=1)
    for t in (0, 1, 2, 6, 7, 8, 9, 10, 12):
        assert tokens[t] == best[t]
    assert tokens[11] == V - 1 and tokens[3] == 0 and tokens[15] == 0


@pytest.mark.parametrize("V", [3, 4, 8, 17, 32, 48, 1000, 5000, 70001])
def test_equal_logits(V):
    """Ties: weights of 1, whose sums are exact, so that every border is; the lowest
    indices are kept."""
    announce(f"sample, equal logits, {V}")
    for xt in ("f32", "bf16"):
        logits, values = _put(np.full((4, V), -3.25), _dtype(xt))
        for rule in (dict(), dict(top_k=[1, 2, V // 2 + 1, V - 1]), dict(top_p=[0.5, 0.25, 0.75, 1 / 1024]), dict(min_p=[1.0] * 4),
                     dict(top_k=[2, V - 1, V // 2 + 1, 3], top_p=[0.5, 0.25, 0.75, 0.5])):
            for u in ([0.0, 0.25, 0.5, 0.75], [1 - 2.0 ** -24] * 4):
                _check(logits, values, u, exact=True, **rule)
        two = values.copy()                      # two levels of ties, the cut among the lower ones
        two[:, ::3] = -2.25
        logits, values = _put(two, _dtype(xt))
        for k in (1, (V + 2) // 3, (V + 2) // 3 + 1, max(1, V - 1)):
            _check(logits, values, [0.1, 0.4, 0.6, 0.9], exact=True, top_k=[k] * 4)
        _check(logits, values, [0.1, 0.4, 0.6, 0.9], top_p=[0.77, 0.3, 0.95, 0.61], exact=V < 100)


def test_masks():
    """Tokens ruled out by -inf or the type's lowest value, rows of nothing else, rows
    with NaN or +inf, choices that are NaN."""
    rng = np.random.default_rng(5)
    V = 3001
    for xt, low in (("f32", np.finfo(np.float32).min), ("bf16", -3.3895e38), ("f16", -65504.0)):
        announce(f"sample, masks, {xt}")
        for mask in (-np.inf, low):
            x = _logits(rng, 6, V)
            x[0, :] = mask
            x[1, 1:] = mask
            x[2, :-1] = mask
            x[3, rng.random(V) < 0.9] = mask
            x[4, : V // 2] = mask
            x[5, ::2] = mask
            logits, values = _put(x, _dtype(xt), 1, 1)
            for rule in (dict(), dict(top_k=[2000] * 6), dict(top_k=[20] * 6), dict(top_p=[0.9] * 6), dict(min_p=[0.01] * 6),
                         dict(top_k=[2500] * 6, top_p=[0.97] * 6)):
                tokens = _check(logits, values, rng.random(6), exact=True, **rule)
                assert tokens[1] == 0 and tokens[2] == V - 1
                assert mask != -np.inf or tokens[0] == -1
        x = _logits(rng, 6, V)
        x[0, 17], x[1, V - 1], x[2, 5], x[3, 0] = np.nan, np.nan, np.inf, np.nan
        x[3, 1:] = -np.inf
        logits, values = _put(x, _dtype(xt))
        for rule in (dict(), dict(top_k=[9] * 6), dict(top_p=[0.5] * 6), dict(temperature=[0.0] * 6)):
            tokens = _check(logits, values, rng.random(6), **rule)
            assert np.all(tokens[:4] == -1) and np.all(tokens[4:] >= 0)
    good, nan = np.full(6, 0.5), np.array([0.5, np.nan, 0.5, 0.5, 0.5, 0.5])
    x, values = _put(_logits(rng, 6, V), _dtype("f32"))
    for rule in (dict(temperature=nan), dict(top_p=nan), dict(min_p=nan)):
        assert _check(x, values, good, **rule)[1] == -1
    assert _check(x, values, nan)[1] == -1


@pytest.mark.parametrize("T", [40, 300])
@pytest.mark.parametrize("xt", ["f32", "bf16"])
def test_lists_of_every_length(T, xt):
    """Lists of tens to thousands of tokens near the cuts, spread, close together and with
    many equal ones, in few and in many rows; the allowed ones at one end, scattered, and
    fewer than top_k, with others so far below that they have hardly a weight, or none."""
    rng = np.random.default_rng(T)
    V = 6000
    for spread in (0.01, 0.3, 2.0):
        x = spread * rng.standard_normal((T, V))
        x[1::4] = np.round(x[1::4] * 8) / 8
        x[2::4, 1500:] -= rng.choice([40.0, 300.0, 2000.0, np.inf], (len(x[2::4]), 1))
        x[3::4, rng.random(V) < 0.7] = -np.inf
        logits, values = _put(x, _dtype(xt))
        for rule in (dict(top_p=rng.uniform(0.02, 0.999, T)), dict(top_k=rng.integers(1, V, T)), dict(min_p=rng.uniform(0.01, 0.99, T)),
                     dict(top_k=rng.integers(100, 4000, T), top_p=rng.uniform(0.1, 0.99, T)), dict(top_k=np.full(T, 1600)),
                     dict(top_k=np.full(T, 5000), top_p=rng.uniform(0.5, 0.99, T))):
            announce(f"sample, lists, {T} rows {xt} spread {spread} {list(rule)}")
            _check(logits, values, rng.random(T), exact=True, **rule)


@pytest.mark.parametrize("V", [1, 20, 300, 2000, 20001, 70001])
def test_whole_multiples_of_the_temperature(V):
    """Logits k times the temperature, exactly: their quotients round up to whole numbers
    as often as down. Few in a row, so that each counts; large ones, near and far from
    each other; every weight is known by k alone."""
    rng = np.random.default_rng(V)
    T = 128 if V <= 2000 else 12
    temperature = rng.uniform(0.02, 3.0, T).astype(np.float32).astype(np.float64)
    for scale in (1, 2 ** 12, 2 ** 30):
        k = (rng.integers(-3, 4, (T, V)) + 8) * scale
        x = (temperature[:, None] * 2.0 ** rng.integers(0, 3, (T, V)) * scale).astype(np.float32)
        x[::2] = (temperature[::2, None] * k[::2]).astype(np.float32)
        logits, values = _put(x.astype(np.float64), _dtype("f32"))
        for rule in (dict(), dict(top_p=[0.8] * T), dict(top_k=[max(1, V // 3)] * T), dict(min_p=[0.01] * T)):
            announce(f"sample, multiples of the temperature, {V}, times {scale}, {rule}")
            _check(logits, values, rng.random(T), temperature=temperature, exact=True, **rule)


@pytest.mark.parametrize("V", [5, 300, 3001, 40000])
def test_lowest_values_at_other_temperatures(V):
    """Rows of the type's lowest value alone (weights of 1 each) and rows masked by it, at
    temperatures whose inverse is rounded, down to the smallest and up to the largest."""
    rng = np.random.default_rng(V + 1)
    for xt, low in (("f32", np.finfo(np.float32).min), ("bf16", -3.3895e38), ("f16", -65504.0)):
        announce(f"sample, lowest values, {xt} {V}")
        temperature = np.array([0.7, 0.3, 1.3, 1e-3, 1e-30, 1e-44, 3e38, 11.0])
        T = len(temperature)
        x = np.full((T, V), low)
        for rows in ("all", "one", "some", "highest"):
            if rows == "one":
                x[:, V // 2] = 1.25
            if rows == "some":
                x[:, ::4] = 1.25
            if rows == "highest":
                x = -x
            logits, values = _put(x, _dtype(xt), 1, 1)
            for rule in (dict(), dict(top_k=[max(1, V // 8)] * T), dict(top_p=[0.3] * T), dict(min_p=[0.5] * T)):
                _check(logits, values, rng.random(T), temperature=temperature, exact=True, **rule)


def test_wide_ranges():
    """Logits that spread over many e-foldings: weights from 1 down to 0 in 64 bits, cuts
    far below the best token, low and high temperatures."""
    rng = np.random.default_rng(8)
    T, V = 5, 9001
    for spread in (1e-3, 30.0, 1e4):
        for xt in ("f32", "bf16"):
            logits, values = _put(spread * rng.standard_normal((T, V)), _dtype(xt))
            for temperature in (0.05, 1.0, 40.0, 1e6, 1e38):
                announce(f"sample, spread {spread} {xt} temperature {temperature}")
                for rule in (dict(top_k=[5, 100, 1100, 5000, 9000]), dict(top_p=[0.5, 0.9, 0.999, 0.999999, 1 - 2.0 ** -24]),
                             dict(top_k=[5, 100, 1100, 5000, 9000], top_p=[0.9, 0.99, 0.9, 0.99, 0.5])):
                    _check(logits, values, rng.random(T), temperature=[temperature] * T, exact=spread == 1e-3 or temperature == 1e38, **rule)


def test_shares_of_the_draws():
    """Evenly spaced u draw every token as often as its probability says, within one
    draw at either end of its interval."""
    import torch
    rng = np.random.default_rng(2)
    V, n = 50, 4000
    x = rng.standard_normal(V)
    logits = torch.as_tensor(np.tile(x, (n, 1)), device=device()).float()
    p = np.exp(logits[0].double().cpu().numpy())
    order = np.argsort(-p)[:20]
    q = np.zeros(V)
    q[order] = p[order] / p[order].sum()
    announce("sample, shares of the draws")
    tokens, _ = _call(logits, (np.arange(n) + 0.5) / n, top_k=np.full(n, 20))
    assert np.all(np.abs(np.bincount(tokens, minlength=V) - n * q) <= 1.0)


def test_many_rows_and_types_of_tokens():
    """More rows than a launch has workgroups; int64 tokens; the same draws again; one
    row among others is one row alone."""
    import torch
    rng = np.random.default_rng(4)
    T, V = 9000, 33
    logits, values = _put(_logits(rng, T, V), _dtype("bf16"), 1, 1)
    u = rng.random(T)
    announce("sample, many rows")
    tokens = _check(logits, values, u, top_p=np.full(T, 0.9))
    again, _ = _call(logits, u, top_p=np.full(T, 0.9), wide=True)
    assert again.dtype == np.int64 and np.array_equal(tokens, again)
    alone, _ = _call(logits[4321:4322], u[4321:4322], top_p=np.full(1, 0.9))
    assert alone[0] == tokens[4321]


def test_replayed_from_a_graph():
    import torch
    from paper_2606_06742_amd import kmpath as km
    rng = np.random.default_rng(6)
    T, V = 5, 40000
    logits, _ = _put(_logits(rng, T, V), torch.bfloat16)
    f = lambda a: torch.as_tensor(a, dtype=torch.float32, device=device())
    u, p = f(rng.random(T)), f(np.full(T, 0.93))
    k = torch.tensor([0, 10, 3000, 0, 40], dtype=torch.int32, device=device())
    ws = torch.empty(km.kmp_sample_tokens_workspace_bytes(T, V), dtype=torch.uint8, device=device())
    out = [(torch.empty(T, dtype=torch.int32, device=device()), torch.empty(T, device=device())) for _ in range(2)]
    call = lambda o, w: km.kmp_sample_tokens(logits, u, o[0], top_k=k, top_p=p, logp=o[1], workspace=w)
    call(out[0], ws)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        call(out[0], ws)
    for i in range(5):
        announce(f"sample replay {i}")
        u.copy_(f(rng.random(T)))
        logits.mul_(0.9)
        g.replay()
        torch.cuda.synchronize()
        call(out[1], torch.empty_like(ws))
        assert torch.equal(out[0][0], out[1][0]) and torch.equal(out[0][1], out[1][1])

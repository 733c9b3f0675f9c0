"""Tokens drawn from vocabularies beyond 2^20 tokens and from more rows than a launch has
workgroups. The longest rows hold two values, 0 and a: the running sums of their weights
1 and w = exp(a) are known in closed form, so that the drawn token is, too. Choices are
taken whose border lies 0.02 to 0.1 tokens from the drawn one. Bound: a weight is within
2^-44 of its size, sums over segments add whole numbers, a lane adds at most 2^13 weights of
one segment of 2^22, and 2^7 additions follow, each within 2^-53 of the sum: 2^-16 + 2^-18 +
2^-18 tokens of 2^28. A cut among equal weights is found by whole numbers in steps of 2^-37
for 2^30 tokens: 2^-8 tokens."""
import numpy as np
import pytest

from oracle import operators as OO
from tests.gpu_common import announce, device
from tests.test_gpu_operators import _dtype, _put
from tests.test_gpu_sample import _call, _check, _logits

pytestmark = pytest.mark.gpu


def _drawn(logits, values, u, **rules):
    """The oracle's tokens, where none of its comparisons is nearer than what the sums are
    off by: weights within 2^-44, V / 512 of them added by a lane at most, and 2^7 additions
    of those, each within 2^-53 of the sum, on both sides."""
    f = lambda a: np.asarray(a, np.float32).astype(np.float64)
    te, le, margin = OO.sample_tokens(values, f(u), **{k: (v if k == "top_k" else f(v)) for k, v in rules.items()})
    tokens, logp = _call(logits, u, **rules)
    off = 2.0 ** -44 + (values.shape[1] / 512 + 2 ** 7) * 2.0 ** -53
    assert np.all(margin > 2 * off), margin
    assert np.array_equal(tokens, te), (tokens, te)
    assert np.all(np.abs(logp - le) <= 2.0 ** -24 * np.abs(le) + 2 * off)


@pytest.mark.parametrize("xt,V", [("bf16", 2 ** 20 + 1), ("f32", 2 ** 20 + 1), ("bf16", 2200003), ("f32", 2200003)])
def test_segments_of_more_elements(xt, V):
    rng = np.random.default_rng(V)
    logits, values = _put(_logits(rng, 2, V), _dtype(xt), 3, 1)
    for rule in (dict(), dict(top_p=[0.9, 0.6]), dict(top_k=[50, 70000]), dict(top_k=[3000, 100], min_p=[1e-3, 0.02]),
                 dict(top_k=[200, 900000], top_p=[0.8, 0.99]), dict(min_p=[1e-5, 0.05])):
        announce(f"sample {xt} 2 x {V} {rule}")
        _drawn(logits, values, rng.random(2), **rule)
        _drawn(logits, values, rng.random(2), temperature=[0.6, 1.7], **rule)
    announce(f"sample {xt} 2 x {V}, equal logits")
    logits, values = _put(np.full((2, V), -3.25), _dtype(xt))
    for rule in (dict(), dict(top_k=[V // 2 + 1, V - 1]), dict(top_p=[0.25, 0.75]), dict(min_p=[1.0] * 2)):
        _check(logits, values, [0.375, 1 - 2.0 ** -24], exact=True, **rule)


def _near(rng, place, n):
    """n choices in (0.1, 0.99) of 32 bits at which place() lies 0.02 to 0.1 from a whole number."""
    c = (rng.integers(int(0.1 * 2 ** 24), int(0.99 * 2 ** 24), 20000) / 2.0 ** 24).astype(np.float32).astype(np.float64)
    off = place(c) - np.rint(place(c))
    below, above = c[(off > -0.1) & (off < -0.02)], c[(off > 0.02) & (off < 0.1)]
    assert len(below) >= n // 2 and len(above) >= n // 2
    return np.concatenate([below[:n // 2], above[:n - n // 2]])


@pytest.mark.parametrize("xt,V,a", [("bf16", 2 ** 28 + 12345, -0.0859375), ("bf16", 2 ** 28 + 12345, -0.396484375),
                                    ("f32", 2 ** 27 + 77, -0.046875), ("bf16", 2 ** 24 + 5, -1.5078125)])
def test_draws_from_long_rows(xt, V, a):
    """Half of the row a, then zeros: the segments' sums decide where the draw falls."""
    import torch
    h, w = V // 2, np.exp(a)
    Z = h * w + (V - h)
    place = lambda u: np.where(u * Z < h * w, u * Z / w, h + (u * Z - h * w))
    us = _near(np.random.default_rng(V), place, 16)
    logits = torch.zeros(1, V, dtype=_dtype(xt), device=device())
    logits[0, :h] = a
    assert float(logits[0, 0]) == a
    got = []
    for u in us:
        announce(f"sample {xt} 1 x {V}, halves of {a} and 0, u {u}")
        got.append(int(_call(logits, [u])[0][0]))
    assert np.array_equal(got, np.floor(place(us)).astype(np.int64)), np.array(got) - np.floor(place(us))


def test_cuts_of_long_rows():
    """2^28 zeros, then -3.84: the shortest run that reaches top_p ends among the latter,
    and u = 1 draws its last token."""
    import torch
    V, n, a, T = 2 ** 30, 2 ** 28, -3.84375, 8
    w = np.exp(a)
    Z = n + (V - n) * w
    place = lambda p: (p * Z - n) / w
    # (from where the run ends among the second value's tokens on)
    ps = _near(np.random.default_rng(30), lambda p: np.where(p * Z > 1.01 * n, place(p), 0.5), T)
    logits = torch.zeros(T, V, dtype=torch.bfloat16, device=device())
    logits[:, n:] = a
    assert float(logits[0, n]) == a
    announce(f"sample bf16 {T} x {V}, top-p {ps}")
    tokens, _ = _call(logits, np.ones(T), top_p=ps)
    want = n + np.ceil(place(ps)).astype(np.int64) - 1
    assert np.array_equal(tokens, want), tokens - want


def test_more_rows_than_workgroups():
    """Launches have up to 65535 workgroups across the rows: each takes more than one."""
    T, V = 66007, 37
    rng = np.random.default_rng(8)
    for xt in ("f32", "bf16"):
        announce(f"sample {xt} {T} x {V}")
        logits, values = _put(_logits(rng, T, V), _dtype(xt), 1, 1)
        temperature = np.where(rng.random(T) < 0.1, 0.0, 0.5 + rng.random(T))
        _check(logits, values, rng.random(T), temperature=temperature, top_k=rng.integers(0, V, T).astype(np.int32),
               top_p=rng.uniform(0.5, 1.2, T), min_p=np.where(rng.random(T) < 0.5, 0.01, 0.0), exact=True)

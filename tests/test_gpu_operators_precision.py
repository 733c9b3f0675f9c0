"""How near the operators come to 64 bits: bounds of the size of the errors that
these kernels should make, against the worst-case bounds of
tests/test_gpu_operators.py, which a kernel that loses some digits would meet.

A sum's roundings are taken as independent, each uniform within u of the partial
sum it rounds: n in a row have a standard deviation of at most u sqrt(n / 3) of the
sum of the terms' sizes, and 8 standard deviations are allowed. n is what one
thread adds (a row's length over the threads that share it) and the tree over them
(at most 16 levels of wavefronts, workgroup and segments)."""
import numpy as np
import pytest

from oracle import operators as OO
from tests.gpu_common import announce, device
from tests.test_gpu_operators import EPS, SHAPES, TINY, U, _dtype, _hidden, _norm_inputs, _np, _put

pytestmark = pytest.mark.gpu


def _spread(n, u):
    return 8.0 * u * np.sqrt((n + 16) / 3.0)


@pytest.mark.parametrize("xt", ["f64", "f32", "bf16", "f16"])
@pytest.mark.parametrize("rows,d", [(64, 100), (50, 1000), (40, 4096), (30, 12000), (20, 40009), (5, 300001)])
def test_layer_norm_precision(xt, rows, d):
    """Rows in registers: at most 32 elements a thread. Longer ones: 1024 threads,
    vectors of up to 8. mu within the sum's spread of mean |x|, rstd within half of
    it and 8 u (quotient, root, products), y then by |g| (rstd dmu + |xh| drstd) and
    4 roundings."""
    import torch
    from paper_2606_06742_amd import kmpath as km
    announce(f"layer norm precision {xt} {rows} x {d}")
    u, uo = U["f64" if xt == "f64" else "f32"], U[xt]
    rng = np.random.default_rng(rows + d)
    x, xv, g, gv, b, bv = _norm_inputs(rng, rows, d, xt, xt, 0, 0)
    st = torch.float64 if xt == "f64" else torch.float32
    y, mean, rstd = torch.empty_like(x), *(torch.empty(rows, dtype=st, device=device()) for _ in "mr")
    km.kmp_layer_norm(x, g, b, EPS, y, mean=mean, rstd=rstd)
    ye, me, re = OO.layer_norm(xv, gv, bv, EPS)
    e = _spread(max(32, d / 1024 + 8), u)
    dmu = e * np.abs(xv).mean(axis=1) + u * np.abs(me)
    drs = e + 8 * u + (dmu * re) ** 2
    assert np.all(np.abs(_np(mean) - me) <= dmu)
    assert np.all(np.abs(_np(rstd) / re - 1.0) <= drs)
    xh = np.abs((xv - me[:, None]) * re[:, None])
    bound = np.abs(gv) * ((dmu * re)[:, None] + xh * drs[:, None]) + 4 * u * (np.abs(bv) + np.abs(ye))
    assert np.all(np.abs(_np(y) - ye) <= bound + (uo if uo != u else 0) * (np.abs(ye) + bound) + TINY[xt])


@pytest.mark.parametrize("xt", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("T,V", [(64, 1003), (32, 9001), (8, 40009), (3, 131101), (520, 50021)])
def test_token_logprobs_precision(xt, T, V):
    """exp(x - m) is in error by u of the difference d for the subtraction, for the
    product with log2 e and for that constant, and by 2 u itself: 3 d + 2, at most,
    in units of u; scaling to a later maximum the same way (3 R for all of an
    element's scalings, R the range that matters). With D = sum p d, D2 = sum p d^2:
    log s within 3 D + 3 R' + 8 and the sum's spread (three roundings a level), where
    R' = R weighted by how much of s was scaled, at most D + 1; the entropy's sum u / s
    by the same relative to (1 + D), and 3 D2 more."""
    import torch
    from paper_2606_06742_amd import kmpath as km
    announce(f"token logprobs precision {xt} {T} x {V}")
    u = U["f32"]
    rng = np.random.default_rng(T + V)
    a = 2.0 * rng.standard_normal((T, V))
    a[np.arange(T), rng.integers(0, V, T)] += 9.0
    tok = rng.integers(0, V, T)
    x, xv = _put(a, _dtype(xt), 0, 0)
    f = lambda *s: torch.empty(*s, device=device())
    logp, H = f(T), f(T)
    ws = torch.empty(km.kmp_token_logprobs_workspace_bytes(T, V, 0), dtype=torch.uint8, device=device())
    km.kmp_token_logprobs(x, torch.as_tensor(tok, device=device()), logp, entropy=H, workspace=ws)
    o = OO.token_logprobs(xv, tok, 0)
    d = xv.max(axis=1)[:, None] - xv
    p = np.exp(-d)
    p /= p.sum(axis=1, keepdims=True)
    D, D2, logs = (p * d).sum(axis=1), (p * d * d).sum(axis=1), o["stats"][:, 1]
    e = _spread(3 * (V / 256 + 16), u)
    lse = e + u * (6 * D + 11 + 2 * logs)
    assert np.all(np.abs(_np(logp) - o["logp"]) <= lse + 2 * u * np.abs(o["logp"])), np.max(np.abs(_np(logp) - o["logp"]) / lse)
    ent = e * (1 + D) + u * ((6 * D + 11) * (1 + D) + 3 * D2 + 4 * logs)
    assert np.all(np.abs(_np(H) - o["entropy"]) <= ent + 2 * u * o["entropy"])


@pytest.mark.parametrize("xt", ["f32", "bf16", "f16"])
def test_quantize_rows_against_the_quotient(xt):
    """x 127 / a in 64 bits, a the row's largest |x|: three roundings (1 / a, times
    127, times x; the lift of tiny rows is exact) of a number of at most 127, then
    the nearest whole one. The scale is one quotient."""
    import torch
    from paper_2606_06742_amd import kmpath as km
    for rows, d, pad, off in SHAPES:
        announce(f"quantize against the quotient {xt} {rows} x {d}")
        rng = np.random.default_rng(rows * 13 + d)
        low, high = (-30, 30) if xt != "f16" else (-2, 3)
        a = _hidden(rng, rows, d) * 10.0 ** rng.integers(low, high, rows)[:, None]
        x, xv = _put(a, _dtype(xt), pad, off)
        q, scale = torch.empty(rows, d, dtype=torch.int8, device=device()), torch.empty(rows, device=device())
        km.kmp_quantize_rows(x, q, scale)
        most = np.abs(xv).max(axis=1)
        want = xv * (127.0 / np.where(most > 0, most, 1.0))[:, None]
        assert np.all(np.abs(_np(q) - want) <= 0.5 + 127 * 3.01 * U["f32"]), (rows, d)
        assert np.all(np.abs(_np(scale) - most / 127.0) <= U["f32"] * most / 127.0 + 2.0 ** -149), (rows, d)

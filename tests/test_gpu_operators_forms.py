"""The operators' kernels beyond one round of a workgroup and beyond one launch:
every register form of the layer norm's two-launch backward pass over every pair
of types, rows that a workgroup takes one after the other, more tokens than a
grid's second dimension holds. Against oracle/operators.py (64 bits) with the
bounds of tests/test_gpu_operators.py, and bit by bit against the same rows in
calls of their own."""
import numpy as np
import pytest

from oracle import operators as OO
from tests.gpu_common import announce, device
from tests.test_gpu_operators import EPS, PAIRS, TINY, U, _dtype, _hidden, _norm_bound, _norm_inputs, _np, _put

pytestmark = pytest.mark.gpu

SIZE = {"f64": 8, "f32": 4, "bf16": 2, "f16": 2}
# rows, 16-byte vectors in a row (the last one not whole): threads x vectors a
# thread 32 x 1, 64 x 1, 64 x 2, 256 x 1, 256 x 2, 512 x 2, 512 x 4, none; all past
# the sizes that take one launch, rows that do not fill the last workgroup
BACKWARD = [(2051, 20), (2053, 50), (2055, 100), (1501, 200), (701, 400), (601, 900), (401, 1500), (301, 2100), (2055, 1)]


@pytest.mark.parametrize("xt,wt", PAIRS)
def test_layer_norm_backward_in_two_launches(xt, wt):
    import torch
    from paper_2606_06742_amd import kmpath as km
    u, uo, uw = U["f64" if xt == "f64" else "f32"], U[xt], U[wt]
    st = torch.float64 if xt == "f64" else torch.float32
    for rows, nv in BACKWARD:
        d = nv * (16 // SIZE[xt]) - 1
        size = rows * d * SIZE[xt]
        assert size > 8 << 20 or rows > 2048 or (rows > 512 and size > 4 << 20)
        announce(f"layer norm backward {xt} weights {wt} {rows} x {d}")
        rng = np.random.default_rng(rows + d)
        x, xv, g, gv, b, _ = _norm_inputs(rng, rows, d, xt, wt, 3, 1)
        dy, dyv = _put(rng.standard_normal((rows, d)) + 0.1, _dtype(xt), 1, 0)
        _, me, re = OO.layer_norm(xv, gv, 0 * gv, EPS)
        mean, rstd = (torch.as_tensor(v, device=device()).to(st) for v in (me, re))
        mk, rk = _np(mean), _np(rstd)
        ws = torch.empty(km.kmp_layer_norm_workspace_bytes(rows, d, _dtype(xt)), dtype=torch.uint8, device=device())
        ws.fill_(255)                            # NaN: every partial sum is written before it is read
        dx, _ = _put(np.zeros((rows, d)), _dtype(xt), 2, 1)
        dg, db = torch.full_like(g, float("nan")), torch.full_like(g, float("nan"))
        km.kmp_layer_norm_backward(dy, x, g, mean, rstd, dx, dg, db, ws)
        dxe, dge, dbe = OO.layer_norm_backward(dyv, xv, gv, mk, rk)
        xh, w, c = np.abs((xv - mk[:, None]) * rk[:, None]), np.abs(dyv * gv), d / 64 + 16
        bound = u * rk[:, None] * ((c + 16) * (w.mean(axis=1)[:, None] + 2 * xh * (w * xh).mean(axis=1)[:, None]) + 8 * w)
        assert np.all(np.abs(_np(dx) - dxe) <= bound + (uo if uo != u else 0) * (np.abs(dxe) + bound) + 2 * u * np.abs(dxe) + TINY[xt]), (rows, d)
        for got, want, size in ((dg, dge, np.abs(dyv) * xh), (db, dbe, np.abs(dyv))):
            bound = (rows + 16) * u * size.sum(axis=0)
            assert np.all(np.abs(_np(got) - want) <= bound + (uw if uw != u else 0) * (np.abs(want) + bound) + TINY[wt]), (rows, d)
        # again, and in parts: the same bits
        for parts in ((True, True, True), (True, False, False), (False, True, False), (False, False, True)):
            outs = [torch.full_like(t, float("nan")) if p else None for p, t in zip(parts, (dx, dg, db))]
            ws.fill_(255)
            km.kmp_layer_norm_backward(dy, x, g, mean, rstd, *outs, ws if any(parts[1:]) else None)
            assert all(o is None or torch.equal(o, t) for o, t in zip(outs, (dx, dg, db))), (rows, d, parts)
        # without weights they are ones
        dx1, dx2 = torch.empty_like(dx), torch.empty_like(dx)
        km.kmp_layer_norm_backward(dy, x, None, mean, rstd, dx1, None, None, None)
        km.kmp_layer_norm_backward(dy, x, torch.ones_like(g), mean, rstd, dx2, None, None, None)
        assert torch.equal(dx1, dx2)


# rows, 16-byte vectors in a row: a grid of 2048 workgroups takes 8 rows of up to 32
# vectors at a time, 4 of up to 128, one of more; further rows in further rounds, the
# last of them not whole. The last two: rows longer than the registers.
ROUNDS = [(16395, 20), (16384 * 2 + 3, 32), (8199, 50), (8201, 100), (4099, 200), (6151, 400), (2049, 900), (2051, 1500),
          (2050, 3000), (2049, 4200)]


@pytest.mark.parametrize("xt", ["f64", "f32", "bf16", "f16"])
def test_layer_norm_and_8_bits_over_many_rounds(xt):
    """Every row against the same row in calls of 512 rows (one round each), and
    rows of every round against the oracle."""
    import torch
    from paper_2606_06742_amd import kmpath as km
    u, uo = U["f64" if xt == "f64" else "f32"], U[xt]
    st = torch.float64 if xt == "f64" else torch.float32
    gen = torch.Generator(device="cuda")
    gen.manual_seed(9)
    for rows, nv in ROUNDS:
        d = nv * (16 // SIZE[xt]) - 1
        announce(f"layer norm, 8 bits {xt} {rows} x {d}")
        # every row has a scale and an offset of its own; gaps of NaN
        buf = torch.full((rows, d + 5), float("nan"), dtype=_dtype(xt), device=device())
        x = buf[:, :d]
        x.copy_(torch.randn(rows, d, generator=gen, device=device()) * (0.5 + torch.rand(rows, 1, generator=gen, device=device()))
                + torch.randn(rows, 1, generator=gen, device=device()))
        g, b = ((torch.randn(d, generator=gen, device=device()) * 0.2 + o).to(_dtype(xt)) for o in (1.0, 0.0))

        def norm(x):
            y, mean, rstd = torch.empty(x.shape[0], d, dtype=x.dtype, device=device()), *(torch.empty(x.shape[0], dtype=st, device=device()) for _ in "mr")
            km.kmp_layer_norm(x, g, b, EPS, y, mean=mean, rstd=rstd)
            return y, mean, rstd

        def norm_bytes(x):
            q, s = torch.empty(x.shape[0], d + 1, dtype=torch.int8, device=device())[:, :d], torch.empty(x.shape[0], device=device())
            km.kmp_layer_norm(x, g, b, EPS, q, scale=s)
            return q, s

        def quantize(x):
            q, s = torch.empty(x.shape[0], d, dtype=torch.int8, device=device()), torch.empty(x.shape[0], device=device())
            km.kmp_quantize_rows(x, q, s)
            return q, s

        calls = [norm] if xt == "f64" else [norm, norm_bytes, quantize]
        some = np.unique(np.r_[0:3, rows // 2, 2047:2051, 8191:8195, 16383:16387, rows - 3:rows])
        some = some[some < rows]
        pick = torch.as_tensor(some, device=device())
        xv, gv, bv = _np(x[pick]), _np(g), _np(b)
        for f in calls:
            whole = f(x)
            parts = zip(*(f(x[i:i + 512]) for i in range(0, rows, 512)))
            assert all(torch.equal(w, torch.cat(p)) for w, p in zip(whole, parts)), (f.__name__, rows, d)
            if f is norm:
                ye, me, re = OO.layer_norm(xv, gv, bv, EPS)
                bound = _norm_bound(xv, gv, bv, ye, me, re, u)
                assert np.all(np.abs(_np(whole[0][pick]) - ye) <= bound + (uo if uo != u else 0) * (np.abs(ye) + bound) + TINY[xt])
            elif f is quantize:
                qe, se = OO.quantize_rows(xv)
                assert np.array_equal(whole[0][pick].cpu().numpy(), qe) and np.array_equal(whole[1][pick].cpu().numpy(), se)


@pytest.mark.parametrize("xt", ["f32", "bf16"])
def test_token_logprobs_of_more_rows_than_a_grid_holds(xt):
    """65535 rows in a grid's second dimension, the rest in further rounds: rows
    that repeat with an odd period have the same bits everywhere."""
    import torch
    from paper_2606_06742_amd import kmpath as km
    rng = np.random.default_rng(4)
    for V, top in ((5, 2), (43, 7)):
        P, T = 701, 2 * 65535 + 77
        announce(f"token logprobs {xt} {T} x {V}")
        base, basev = _put(rng.standard_normal((P, V)) * 2.0, _dtype(xt))
        tok = rng.integers(-1, V, P)
        gv, hv = rng.standard_normal(P), rng.standard_normal(P)
        at = torch.arange(T, device=device()) % P
        put = lambda a, t: torch.as_tensor(a, device=device()).to(t)
        tokens, g, h = put(tok, torch.int64), put(gv, torch.float32), put(hv, torch.float32)

        def call(x, tokens, g, h):
            n = x.shape[0]
            f = lambda *s: torch.full(s, float("nan"), device=device())
            lp, H, st, tl, dx = f(n), f(n), f(n, 2), f(n, top), torch.full_like(x, float("nan"))
            ti = torch.full((n, top), -7, dtype=torch.int32, device=device())
            ws = torch.empty(km.kmp_token_logprobs_workspace_bytes(n, V, top), dtype=torch.uint8, device=device())
            km.kmp_token_logprobs(x, tokens, lp, entropy=H, stats=st, top_id=ti, top_logp=tl, workspace=ws)
            km.kmp_token_logprobs_backward(x, tokens, st, g, dx, entropy=H, dentropy=h)
            return lp, H, st, ti, tl, dx

        few = call(base, tokens, g, h)
        many = call(base[at], tokens[at], g[at], h[at])
        assert all(torch.equal(m, f[at]) for m, f in zip(many, few))
        o = OO.token_logprobs(basev, tok, top)
        assert np.array_equal(few[3].cpu().numpy(), o["top_id"])
        # at most 43 terms by as many threads: 64 u as in the tests of other sizes
        assert np.all(np.abs(_np(few[0]) - o["logp"]) <= 128 * U["f32"] * (1 + np.abs(o["logp"])))
        assert np.all(np.abs(_np(few[1]) - o["entropy"]) <= 512 * U["f32"] * (1 + o["entropy"]))


@pytest.mark.parametrize("xt", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("T,V", [(1, 1), (5, 100), (3, 4097), (300, 1003), (2, 40009)])
def test_gradient_of_the_entropy_alone(xt, T, V):
    """No tokens and no dlogp: -h p (log p + H); a row without a possible token has
    none, one with NaN is NaN. p within (4 |lp| + 2 log s + 16) u, as with both terms."""
    import torch
    from paper_2606_06742_amd import kmpath as km
    announce(f"gradient of the entropy {xt} {T} x {V}")
    rng = np.random.default_rng(T * 31 + V)
    a = 2.0 * rng.standard_normal((T, V))
    if V > 4:
        a[:, rng.integers(0, V, V // 8)] = -np.inf
    if T > 2:
        a[1] = -np.inf
        a[2, V // 2] = np.nan
    x, xv = _put(a, _dtype(xt), 3, 1)
    f = lambda *s: torch.empty(*s, device=device())
    H, st = f(T), f(T, 2)
    ws = torch.empty(km.kmp_token_logprobs_workspace_bytes(T, V, 0), dtype=torch.uint8, device=device())
    km.kmp_token_logprobs(x, None, None, entropy=H, stats=st, workspace=ws)
    h = torch.as_tensor(rng.standard_normal(T), device=device()).float()
    dx, _ = _put(np.zeros((T, V)), _dtype(xt), 2, 1)
    km.kmp_token_logprobs_backward(x, None, st, None, dx, entropy=H, dentropy=h)
    sv, Hv, hv = _np(st), _np(H), _np(h)
    want = OO.token_logprobs_backward(xv, None, sv, None, Hv, hv)
    got = _np(dx)
    assert np.array_equal(np.isnan(got), np.isnan(want))
    with np.errstate(invalid="ignore"):
        lp = np.where(xv > -np.inf, (xv - sv[:, :1]) - sv[:, 1:], 0.0)
        p = np.where(xv > -np.inf, np.exp(lp), 0.0)
        term = p * np.abs(hv)[:, None] * (np.abs(lp) + np.abs(Hv)[:, None])
        bound = U["f32"] * term * (4 * np.abs(lp) + 2 * np.abs(sv[:, 1:]) + 16) + 2.0 ** -120
        ok = np.abs(got - want) <= bound + (U[xt] if xt != "f32" else 0) * (np.abs(want) + bound) + TINY[xt]
    assert np.all(ok | np.isnan(want) | (want == got))
    km.kmp_token_logprobs_backward(x, None, st, None, x, entropy=H, dentropy=h)      # in place
    assert torch.equal(x.nan_to_num(7.0), dx.nan_to_num(7.0))

"""Layer norm, 8-bit products and token log probabilities on the GPU against
oracle/operators.py (64 bits), over types, sizes around every form's borders,
strides, unaligned rows, masks and non-finite values.

Bounds. u is the unit roundoff of the arithmetic (2^-24, 2^-53 for doubles), uo
that of the output type. A sum of d terms over at least 64 lanes is taken to be
in error by at most (d/64 + 16) u times the sum of the terms' sizes (each lane's
running sum, then a tree); a product, quotient, root or exponential adds a few u.
The bounds below are first-order sums of such terms, written beside each test."""
import ctypes as C

import numpy as np
import pytest

from oracle import operators as OO
from tests.gpu_common import announce, device

pytestmark = pytest.mark.gpu

EPS = 1e-5
U = {"f64": 2.0 ** -53, "f32": 2.0 ** -24, "bf16": 2.0 ** -8, "f16": 2.0 ** -11}
TINY = {"f64": 0.0, "f32": 2.0 ** -149, "bf16": 2.0 ** -133, "f16": 2.0 ** -25}


def _dtype(name):
    import torch
    return {"f64": torch.float64, "f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}[name]


def _put(a, dtype, pad=0, off=0):
    """(tensor, its values in 64 bits): a's rows `pad` elements further apart
    than they are long, the first `off` elements into its memory; the gaps hold
    NaN (or -128), which nothing may read into a result."""
    import torch
    t = torch.as_tensor(np.asarray(a, dtype=np.float64) if np.asarray(a).dtype != np.int8 else a).to(device()).to(dtype)
    r, c = t.shape
    fill = -128 if dtype == torch.int8 else float("nan")
    buf = torch.full((r * (c + pad) + off,), fill, dtype=dtype, device=device())
    v = buf[off:].view(r, c + pad)[:, :c]
    v.copy_(t)
    return v, v.double().cpu().numpy()


def _np(t):
    return t.double().cpu().numpy()


def _hidden(rng, rows, d):
    return rng.standard_normal((rows, d)) * np.exp(0.5 * rng.standard_normal(d)) + 0.3 * rng.standard_normal(d)


# rows, d, gap between rows, first element's offset: lanes that hold nothing,
# one, several vectors; borders of the forms; odd rows at odd addresses
SHAPES = [(1, 1, 0, 0), (3, 2, 1, 1), (5, 7, 0, 0), (2, 64, 0, 0), (4, 100, 4, 0), (9, 255, 0, 1),
          (3, 257, 3, 0), (2, 511, 0, 0), (2, 513, 0, 0), (7, 1024, 8, 0), (2, 1999, 0, 1), (3, 2048, 0, 0),
          (2, 2056, 0, 0), (1, 4096, 0, 0), (5, 4100, 4, 2), (2, 8192, 0, 0), (2, 8200, 0, 0), (2, 16384, 0, 0),
          (2, 16385, 0, 1), (1, 40009, 0, 0)]
PAIRS = [("f64", "f64"), ("f32", "f32"), ("bf16", "bf16"), ("bf16", "f32"), ("f16", "f16"), ("f16", "f32")]


def _norm_inputs(rng, rows, d, xt, wt, pad, off):
    x, xv = _put(_hidden(rng, rows, d), _dtype(xt), pad, off)
    g, gv = _put(1.0 + 0.2 * rng.standard_normal((1, d)), _dtype(wt))
    b, bv = _put(0.1 * rng.standard_normal((1, d)), _dtype(wt))
    return x, xv, g[0], gv[0], b[0], bv[0]


def _norm_bound(xv, gv, bv, y, mean, rstd, u):
    """|dy| <= |g| (rstd |dmu| + |xh| (relative error of rstd + 3u)) + u (|xh g| + |b| + |y|):
    dmu = c u mean|x|, rstd within (c + 8) u and (dmu rstd)^2, c = d/64 + 16."""
    d = xv.shape[1]
    c = d / 64 + 16
    dmu = (c * u * np.abs(xv).mean(axis=1) * rstd)[:, None]
    xh = np.abs((xv - mean[:, None]) * rstd[:, None])
    return np.abs(gv) * (dmu + xh * ((c + 12) * u + dmu ** 2)) + 4 * u * (np.abs(bv) + np.abs(y))


@pytest.mark.parametrize("xt,wt", PAIRS)
def test_layer_norm_forward_and_backward(xt, wt):
    import torch
    from paper_2606_06742_amd import kmpath as km
    u, uo, uw = U["f64" if xt == "f64" else "f32"], U[xt], U[wt]
    for rows, d, pad, off in SHAPES:
        announce(f"layer norm {xt} weights {wt} {rows} x {d} gap {pad} offset {off}")
        rng = np.random.default_rng(rows * 100003 + d)
        x, xv, g, gv, b, bv = _norm_inputs(rng, rows, d, xt, wt, pad, off)
        y, _ = _put(np.zeros((rows, d)), _dtype(xt), pad, off)
        st = torch.float64 if xt == "f64" else torch.float32
        mean, rstd = torch.empty(rows, dtype=st, device=device()), torch.empty(rows, dtype=st, device=device())
        km.kmp_layer_norm(x, g, b, EPS, y, mean=mean, rstd=rstd)
        ye, me, re = OO.layer_norm(xv, gv, bv, EPS)
        bound = _norm_bound(xv, gv, bv, ye, me, re, u)
        assert np.all(np.abs(_np(y) - ye) <= bound + (uo if uo != u else 0) * (np.abs(ye) + bound) + TINY[xt]), (rows, d)
        c = d / 64 + 16
        dmu = c * u * np.abs(xv).mean(axis=1)
        assert np.all(np.abs(_np(mean) - me) <= dmu + u * np.abs(me))
        assert np.all(np.abs(_np(rstd) / re - 1.0) <= (c + 8) * u + (dmu * re) ** 2)
        # backward, at the statistics that the forward call returned: w within
        # 2u, xh within 2u (x - mu is rounded once), the means within (c + 8) u
        dy, dyv = _put(rng.standard_normal((rows, d)) + 0.1, _dtype(xt), pad, off)
        dx, _ = _put(np.zeros((rows, d)), _dtype(xt), pad, off)
        dg, db = torch.empty_like(g), torch.empty_like(b)
        ws = torch.empty(km.kmp_layer_norm_workspace_bytes(rows, d, _dtype(xt)), dtype=torch.uint8, device=device())
        km.kmp_layer_norm_backward(dy, x, g, mean, rstd, dx, dg, db, ws)
        mk, rk = _np(mean), _np(rstd)
        dxe, dge, dbe = OO.layer_norm_backward(dyv, xv, gv, mk, rk)
        xh = np.abs((xv - mk[:, None]) * rk[:, None])
        w = np.abs(dyv * gv)
        bound = u * rk[:, None] * ((c + 16) * (w.mean(axis=1)[:, None] + 2 * xh * (w * xh).mean(axis=1)[:, None]) + 8 * w)
        assert np.all(np.abs(_np(dx) - dxe) <= bound + (uo if uo != u else 0) * (np.abs(dxe) + bound) + 2 * u * np.abs(dxe) + TINY[xt]), (rows, d)
        for got, want, size in ((dg, dge, np.abs(dyv) * xh), (db, dbe, np.abs(dyv))):
            bound = (rows + 16) * u * size.sum(axis=0)
            assert np.all(np.abs(_np(got) - want) <= bound + (uw if uw != u else 0) * (np.abs(want) + bound) + TINY[wt]), (rows, d)
        # parts alone give the same bits
        dx2, dg2 = torch.empty(rows, d, dtype=x.dtype, device=device()), torch.empty_like(g)
        km.kmp_layer_norm_backward(dy, x, g, mean, rstd, dx2, None, None, None)
        km.kmp_layer_norm_backward(dy, x, g, mean, rstd, None, dg2, None, ws)
        assert torch.equal(dx2, dx) and torch.equal(dg2, dg)


@pytest.mark.parametrize("rows", [1, 31, 700, 2049, 5003])
def test_layer_norm_weight_gradients_over_many_rows(rows):
    """The reduction over rows: counts around its strips, the same bits again."""
    import torch
    from paper_2606_06742_amd import kmpath as km
    for d in (7, 96, 1000, 2500, 7001):
        announce(f"layer norm backward f32 {rows} x {d}")
        rng = np.random.default_rng(rows + d)
        x, xv, g, gv, b, bv = _norm_inputs(rng, rows, d, "f32", "f32", 0, 0)
        dy, dyv = _put(rng.standard_normal((rows, d)), torch.float32)
        _, me, re = OO.layer_norm(xv, gv, bv, EPS)
        mean, rstd = (torch.as_tensor(v, device=device()).float() for v in (me, re))
        ws = torch.empty(km.kmp_layer_norm_workspace_bytes(rows, d, torch.float32), dtype=torch.uint8, device=device())
        outs = []
        for _ in range(2):
            ws.fill_(255)                        # NaN: every partial sum is written before it is read
            dx, dg, db = torch.empty_like(x), torch.empty_like(g), torch.empty_like(b)
            km.kmp_layer_norm_backward(dy, x, g, mean, rstd, dx, dg, db, ws)
            outs.append((dx, dg, db))
        assert all(torch.equal(p, q) for p, q in zip(*outs))
        _, dge, dbe = OO.layer_norm_backward(dyv, xv, gv, _np(mean), _np(rstd))
        xh = np.abs((xv - _np(mean)[:, None]) * _np(rstd)[:, None])
        for got, want, size in ((dg, dge, np.abs(dyv) * xh), (db, dbe, np.abs(dyv))):
            assert np.all(np.abs(_np(got) - want) <= (rows + 16) * U["f32"] * size.sum(axis=0))


# rows too long for registers and rows shorter than a vector, with the sums in a
# launch beside dx and in passes of their own
@pytest.mark.parametrize("xt,rows,d", [("f32", 40, 9001), ("f32", 300, 16500), ("bf16", 60, 16391), ("bf16", 600, 8200),
                                       ("f16", 300, 17000), ("f32", 2500, 3), ("f32", 1000, 3), ("bf16", 3000, 7)])
def test_layer_norm_gradients_of_long_and_tiny_rows(xt, rows, d):
    import torch
    from paper_2606_06742_amd import kmpath as km
    announce(f"layer norm backward {xt} {rows} x {d}")
    u, uo = U["f32"], U[xt]
    rng = np.random.default_rng(rows + d)
    x, xv, g, gv, b, _ = _norm_inputs(rng, rows, d, xt, "f32", 3, 1)
    dy, dyv = _put(rng.standard_normal((rows, d)) + 0.1, _dtype(xt), 1, 0)
    _, me, re = OO.layer_norm(xv, gv, 0 * gv, EPS)
    mean, rstd = (torch.as_tensor(v, device=device()).float() for v in (me, re))
    mk, rk = _np(mean), _np(rstd)
    ws = torch.empty(km.kmp_layer_norm_workspace_bytes(rows, d, _dtype(xt)), dtype=torch.uint8, device=device())
    ws.fill_(255)                                # NaN: every partial sum is written before it is read
    dx, _ = _put(np.zeros((rows, d)), _dtype(xt), 2, 1)
    dg, db = torch.empty_like(g), torch.empty_like(b)
    km.kmp_layer_norm_backward(dy, x, g, mean, rstd, dx, dg, db, ws)
    dxe, dge, dbe = OO.layer_norm_backward(dyv, xv, gv, mk, rk)
    xh, w, c = np.abs((xv - mk[:, None]) * rk[:, None]), np.abs(dyv * gv), d / 64 + 16
    bound = u * rk[:, None] * ((c + 16) * (w.mean(axis=1)[:, None] + 2 * xh * (w * xh).mean(axis=1)[:, None]) + 8 * w)
    assert np.all(np.abs(_np(dx) - dxe) <= bound + (uo if uo != u else 0) * (np.abs(dxe) + bound) + 2 * u * np.abs(dxe) + TINY[xt])
    for got, want, size in ((dg, dge, np.abs(dyv) * xh), (db, dbe, np.abs(dyv))):
        assert np.all(np.abs(_np(got) - want) <= (rows + 16) * u * size.sum(axis=0) + TINY["f32"])
    dx2, dg2 = torch.empty(rows, d, dtype=x.dtype, device=device()), torch.empty_like(g)
    km.kmp_layer_norm_backward(dy, x, g, mean, rstd, dx2, None, None, None)
    km.kmp_layer_norm_backward(dy, x, g, mean, rstd, None, dg2, None, ws)
    assert torch.equal(dx2, dx) and torch.equal(dg2, dg)


def test_layer_norm_gradient_against_differences():
    """64-bit rows: the backward against central differences of the forward.
    Step 1e-4: error 1e-8 times third derivatives (tens), rounding 1e-12."""
    import torch
    from paper_2606_06742_amd import kmpath as km
    announce("layer norm f64 differences")
    rng = np.random.default_rng(8)
    rows, d, h = 2, 11, 1e-4
    x = torch.as_tensor(rng.standard_normal((rows, d)), device=device())
    g, b, dy = (torch.as_tensor(rng.standard_normal(s), device=device()) for s in (d, d, (rows, d)))
    mean, rstd = torch.empty(rows, dtype=torch.float64, device=device()), torch.empty(rows, dtype=torch.float64, device=device())
    y = torch.empty_like(x)

    def f(x_, g_):
        km.kmp_layer_norm(x_, g_, b, 1e-2, y, mean=mean, rstd=rstd)
        return float((y * dy).sum())

    def slope(t, i, call):
        old = float(t[i])
        t[i] = old + h
        up = call()
        t[i] = old - h
        down = call()
        t[i] = old
        return (up - down) / (2 * h)

    f(x, g)
    dx, dg, db = torch.empty_like(x), torch.empty_like(g), torch.empty_like(b)
    ws = torch.empty(km.kmp_layer_norm_workspace_bytes(rows, d, torch.float64), dtype=torch.uint8, device=device())
    km.kmp_layer_norm_backward(dy, x, g, mean, rstd, dx, dg, db, ws)
    for i in np.ndindex(rows, d):
        assert abs(slope(x, i, lambda: f(x, g)) - float(dx[i])) < 1e-5
    for j in range(d):
        assert abs(slope(g, j, lambda: f(x, g)) - float(dg[j])) < 1e-5


def test_layer_norm_edges():
    """No weights; constant and huge rows; NaN and infinity stay in their row;
    no rows: the weight gradients are zero."""
    import torch
    from paper_2606_06742_amd import kmpath as km
    announce("layer norm edges")
    x = torch.full((4, 300), 3.0, device=device())
    x[1] = torch.linspace(-1e18, 1e18, 300)
    x[2, 7] = float("nan")
    x[3, 299] = float("inf")
    y = torch.empty_like(x)
    km.kmp_layer_norm(x, None, None, EPS, y)
    assert bool((y[0] == 0).all()) and bool(torch.isfinite(y[1]).all()) and bool(y[2:].isnan().any(dim=1).all())
    ye = OO.layer_norm(_np(x[1:2]), None, None, EPS)[0]
    assert np.abs(_np(y[1:2]) - ye).max() < 1e-5
    g = torch.ones(5, device=device())
    none = torch.empty(0, 5, device=device())
    dg, db = torch.full_like(g, 7.0), torch.full_like(g, 7.0)
    ws = torch.empty(km.kmp_layer_norm_workspace_bytes(0, 5, torch.float32), dtype=torch.uint8, device=device())
    m = torch.empty(0, device=device())
    km.kmp_layer_norm_backward(none, none, g, m, m, none, dg, db, ws)
    km.kmp_layer_norm(none, g, g, EPS, none)
    assert bool((dg == 0).all()) and bool((db == 0).all())


# ------------------------------------------------------------------ 8 bits
@pytest.mark.parametrize("xt", ["f32", "bf16", "f16"])
def test_quantize_rows_exactly(xt):
    import torch
    from paper_2606_06742_amd import kmpath as km
    for rows, d, pad, off in SHAPES:
        announce(f"quantize {xt} {rows} x {d} gap {pad} offset {off}")
        rng = np.random.default_rng(rows * 7 + d)
        a = _hidden(rng, rows, d) * 10.0 ** rng.integers(-3, 4, rows)[:, None]
        x, xv = _put(a, _dtype(xt), pad, off)
        q, _ = _put(np.zeros((rows, d), np.int8), torch.int8, pad, off)
        scale = torch.empty(rows, device=device())
        km.kmp_quantize_rows(x, q, scale)
        qe, se = OO.quantize_rows(xv)
        assert np.array_equal(q.cpu().numpy(), qe) and np.array_equal(scale.cpu().numpy(), se), (rows, d)


def test_quantize_rows_edges():
    """Zero, tiny, non-finite rows and ties at halves."""
    import torch
    from paper_2606_06742_amd import kmpath as km
    announce("quantize edges")
    for d in (5, 600, 20000):
        a = np.zeros((7, d), np.float32)
        a[1, :2] = 1e-42, -2e-42
        a[2, :3] = 1e-33, -3e-33, 2e-33
        a[3, 0], a[3, 1] = np.inf, 1.0
        a[4, d - 1] = np.nan
        a[5, :5] = 127.0, 0.5, 1.5, -2.5, 126.5
        a[6, 0] = 3.4e38
        x = torch.as_tensor(a, device=device())
        q, scale = torch.empty(7, d, dtype=torch.int8, device=device()), torch.empty(7, device=device())
        km.kmp_quantize_rows(x, q, scale)
        qe, se = OO.quantize_rows(a)
        assert np.array_equal(q.cpu().numpy(), qe) and np.array_equal(scale.cpu().numpy(), se, equal_nan=True)


@pytest.mark.parametrize("xt", ["f32", "bf16", "f16"])
def test_layer_norm_in_8_bits(xt):
    """The scale is a/127 with a within the bound of the norm's values; a
    quantised value times the scale is within half a step (and the bound) of y."""
    import torch
    from paper_2606_06742_amd import kmpath as km
    for rows, d, pad, off in SHAPES:
        announce(f"layer norm in 8 bits {xt} {rows} x {d}")
        rng = np.random.default_rng(rows * 31 + d)
        x, xv, g, gv, b, bv = _norm_inputs(rng, rows, d, xt, xt, pad, off)
        q, _ = _put(np.zeros((rows, d), np.int8), torch.int8, pad, off)
        scale = torch.empty(rows, device=device())
        km.kmp_layer_norm(x, g, b, EPS, q, scale=scale)
        ye, me, re = OO.layer_norm(xv, gv, bv, EPS)
        bound = _norm_bound(xv, gv, bv, ye, me, re, U["f32"])
        s = _np(scale)[:, None]
        assert np.all(np.abs(s[:, 0] * 127 - np.abs(ye).max(axis=1)) <= bound.max(axis=1) + 2.0 ** -22 * s[:, 0] * 127)
        assert np.all(np.abs(_np(q) * s - ye) <= s * (0.5 + 2.0 ** -14) + bound)


# M, N, K: one token, a few, borders of the skinny, small and large tiles, ragged
# everywhere, an empty sum, one slice and a bit
PRODUCTS = [(1, 1, 1), (1, 17, 5), (3, 16, 0), (1, 64, 64), (2, 33, 130), (1, 1000, 4096), (5, 129, 1000), (16, 48, 63),
            (17, 256, 65), (33, 100, 2051), (64, 513, 512), (65, 64, 127), (100, 300, 129), (128, 128, 128),
            (129, 257, 384), (255, 640, 130), (256, 256, 256), (257, 511, 259), (300, 2000, 1000), (520, 1030, 77),
            (1000, 3, 640), (2049, 513, 192),
            (1100, 2100, 200),
            (3500, 3600, 384), (3600, 3500, 130)]      # the larger tiles


def _bytes(rng, r, k):
    a = rng.integers(-127, 128, (r, k)).astype(np.int8)
    if a.size:
        a[rng.integers(0, r), :] = -128           # the type's lowest value is allowed
    return a


@pytest.mark.parametrize("ot", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("pad,off", [(0, 0), (16, 16), (64, 0), (3, 1)])
def test_quantized_product(ot, pad, off):
    """Whole sums are exact, then converted, scaled twice, the bias added: 4
    roundings in 32 bits and the output's."""
    import torch
    from paper_2606_06742_amd import kmpath as km
    for M, N, K in PRODUCTS:
        up = -K % 16 if pad >= 16 else 0           # rows at multiples of 16 bytes
        announce(f"quantized product {ot} {M} x {N} x {K} gap {pad + up} offset {off}")
        rng = np.random.default_rng(M * 1009 + N * 31 + K)
        x, w = _bytes(rng, M, K), _bytes(rng, N, K)
        xq, _ = _put(x, torch.int8, pad + up, off)
        wq, _ = _put(w, torch.int8, pad + up, off)
        xs, ws = rng.uniform(0.001, 0.002, M).astype(np.float32), rng.uniform(0.0005, 0.001, N).astype(np.float32)
        bias = rng.standard_normal(N).astype(np.float32) if (M + N) % 2 else None
        out, _ = _put(np.zeros((M, N)), _dtype(ot), pad, off)
        put = lambda a: None if a is None else torch.as_tensor(a, device=device())
        km.kmp_quantized_product(xq, put(xs), wq, put(ws), out, bias=put(bias))
        p = OO.quantized_product(x, xs, w, ws)
        want = p if bias is None else p + bias
        bound = 4 * U["f32"] * (np.abs(p) + np.abs(want)) + (0 if bias is None else U["f32"] * np.abs(bias))
        uo = U[ot] if ot != "f32" else 0.0
        assert np.all(np.abs(_np(out) - want) <= bound + uo * (np.abs(want) + bound) + TINY[ot]), (M, N, K)


# between the forms' sizes: many tiles of each, slices of 128 bytes from none to more
# than are on their way, with and without a rest
@pytest.mark.parametrize("pad", [0, 1, 16], ids=["packed", "odd", "aligned"])
@pytest.mark.parametrize("M,N", [(33, 70), (40, 8200), (1500, 1500), (1700, 1750)])
def test_quantized_product_slices(M, N, pad):
    import torch
    from paper_2606_06742_amd import kmpath as km
    for K in (5, 127, 128, 130, 256, 300, 384, 515, 640, 777, 1024, 1153, 1290):
        announce(f"quantized product {M} x {N} x {K} gap {pad}")
        g = torch.Generator().manual_seed(M + N + K)
        x, w = (torch.randint(-128, 128, (r, K), dtype=torch.int8, generator=g) for r in (M, N))
        ld = K + (-K % 16 if pad == 16 else pad)
        xq, wq = (torch.full((r, ld), 77, dtype=torch.int8, device=device())[:, :K] for r in (M, N))
        xq.copy_(x)
        wq.copy_(w)
        out = torch.empty(M, N, device=device())
        km.kmp_quantized_product(xq, torch.ones(M, device=device()), wq, torch.ones(N, device=device()), out)
        # below 2^24 in magnitude nearly always; one rounding to 32 bits otherwise
        want = (x.double() @ w.double().T).float()
        assert torch.equal(out.cpu(), want), (M, N, K)


# a tile of 128 for each compute unit at most: a ring of four slices, from none to
# more than it holds
@pytest.mark.parametrize("M,N,Ks", [(1900, 2000, (5, 128, 129, 250, 384, 400, 512, 530, 640, 777, 1025)),
                                    (1300, 1450, (2048, 2177)), (100, 28000, (2048, 2200))])
def test_quantized_product_slices_in_a_ring_of_four(M, N, Ks):
    import torch
    from paper_2606_06742_amd import kmpath as km
    for K in Ks:
        announce(f"quantized product {M} x {N} x {K}")
        g = torch.Generator().manual_seed(M + N + K)
        x, w = (torch.randint(-128, 128, (r, K), dtype=torch.int8, generator=g) for r in (M, N))
        xq, wq = (torch.full((r, K + -K % 16), 77, dtype=torch.int8, device=device())[:, :K] for r in (M, N))
        xq.copy_(x)
        wq.copy_(w)
        out = torch.empty(M, N, device=device())
        km.kmp_quantized_product(xq, torch.ones(M, device=device()), wq, torch.ones(N, device=device()), out)
        # the sums are whole numbers; one rounding to 32 bits
        assert torch.equal(out.cpu(), (x.double() @ w.double().T).float()), (M, N, K)


def test_quantized_product_largest_sums_and_rows():
    """The largest sum that is allowed; NaN scales stay in their row or column."""
    import torch
    from paper_2606_06742_amd import kmpath as km
    K = 131071
    for M in (1, 70):
        announce(f"quantized product {M} x 20 x {K}")
        x = torch.full((M, K), -128, dtype=torch.int8, device=device())
        w = torch.full((20, K), -128, dtype=torch.int8, device=device())
        xs, ws, out = torch.ones(M, device=device()), torch.ones(20, device=device()), torch.empty(M, 20, device=device())
        xs[M - 1] = float("nan")
        ws[3] = float("inf")
        km.kmp_quantized_product(x, xs, w, ws, out)
        fine = out[:M - 1, torch.arange(20, device=device()) != 3]
        assert bool((fine == float(np.float32(16384 * K))).all())
        assert bool(out[M - 1].isnan().all()) and bool(out[:M - 1, 3].isinf().all())


def test_norm_to_product_chain_on_a_side_stream():
    """The 8-bit rows of the norm go straight into the product, on a stream of
    the caller's own."""
    import torch
    from paper_2606_06742_amd import kmpath as km
    announce("norm to product on a side stream")
    rng = np.random.default_rng(12)
    M, K, N = 21, 515, 77
    x, xv, g, gv, b, bv = _norm_inputs(rng, M, K, "bf16", "bf16", 0, 0)
    w, _ = _put(_bytes(rng, N, K), torch.int8, 5)
    ws = torch.full((N,), 0.01, device=device())
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        q, scale = torch.empty(M, K, dtype=torch.int8, device=device()), torch.empty(M, device=device())
        out = torch.empty(M, N, device=device())
        km.kmp_layer_norm(x, g, b, EPS, q, scale=scale, stream=s)
        km.kmp_quantized_product(q, scale, w, ws, out, stream=s)
    s.synchronize()
    want = OO.quantized_product(q.cpu().numpy(), scale.cpu().numpy(), w.cpu().numpy(), ws.cpu().numpy())
    assert np.all(np.abs(_np(out) - want) <= 8 * U["f32"] * np.abs(want))


# ------------------------------------------------- log probabilities of tokens
# T, V, top, gap, offset: less than a vector, one, a lane's, the forms' borders,
# one long row, many rows
LOGITS = [(1, 1, 1, 0, 0), (3, 2, 2, 1, 1), (4, 7, 3, 0, 0), (2, 64, 64, 0, 0), (5, 100, 5, 4, 0), (2, 1000, 20, 0, 1),
          (3, 2047, 1, 0, 0), (2, 2049, 8, 7, 3), (7, 4099, 20, 0, 0), (1, 32000, 20, 0, 0), (2, 40009, 33, 0, 1),
          (1, 131101, 64, 0, 0), (300, 1003, 4, 5, 0), (700, 513, 0, 0, 0), (600, 9001, 5, 0, 0)]


def _logits(rng, T, V):
    x = 2.0 * rng.standard_normal((T, V))
    x[np.arange(T), rng.integers(0, V, T)] += 9.0
    if V > 4:
        x[::3, rng.integers(0, V, V // 8)] = -np.inf
        x[1::4, V // 2:] = -3.0e4                  # nearly ruled out
    tok = rng.integers(0, V, T)
    tok[1::5] = -1
    return x, tok


def _logprob_bounds(xv, o):
    """First-order error of log s (and of log p), and of the entropy. With d =
    m - x_j: exp has relative error (2 d + 4) u, sums (V/64 + 64) u, rescaling by
    exp(m - m') 4 u times the distances (at most the range R that matters)."""
    u, V = U["f32"], xv.shape[1]
    m = xv.max(axis=1)
    with np.errstate(invalid="ignore"):
        d = np.where(xv > -np.inf, m[:, None] - xv, np.inf)
        p = np.exp(-d)
        p /= p.sum(axis=1, keepdims=True)
        dd = np.where(p > 0, d, 0.0)
    D, D2 = (p * dd).sum(axis=1), (p * dd ** 2).sum(axis=1)
    R = np.where(dd < 104, dd, 0.0).max(axis=1)
    logs = np.abs(o["stats"][:, 1])
    lse = u * (V / 64 + 64 + 4 * D + 4 * R + 4 * logs)
    ent = u * ((V / 64 + 64 + 4 * R) * (1 + D) + 4 * D2 + 8 * logs)
    return lse, ent


@pytest.mark.parametrize("xt", ["f32", "bf16", "f16"])
def test_token_logprobs_and_gradient(xt):
    import torch
    from paper_2606_06742_amd import kmpath as km
    u, uo = U["f32"], U[xt]
    for T, V, top, pad, off in LOGITS:
        announce(f"token logprobs {xt} {T} x {V} top {top} gap {pad} offset {off}")
        rng = np.random.default_rng(T * 10007 + V)
        a, tok = _logits(rng, T, V)
        x, xv = _put(a, _dtype(xt), pad, off)
        tokens = torch.as_tensor(tok, device=device())
        if T % 2:
            tokens = tokens.int()
        f = lambda *s: torch.full(s, float("nan"), device=device())
        logp, ent, stats, tl = f(T), f(T), f(T, 2), f(T, top)
        ti = torch.full((T, top), -7, dtype=torch.int32, device=device())
        ws = torch.empty(km.kmp_token_logprobs_workspace_bytes(T, V, top), dtype=torch.uint8, device=device())
        km.kmp_token_logprobs(x, tokens, logp, entropy=ent, stats=stats, top_id=ti, top_logp=tl, workspace=ws)
        o = OO.token_logprobs(xv, tok, top)
        bl, be = _logprob_bounds(xv, o)
        assert np.array_equal(ti.cpu().numpy(), o["top_id"]), (T, V)
        assert np.array_equal(_np(stats)[:, 0], o["stats"][:, 0])
        assert np.all(np.abs(_np(stats)[:, 1] - o["stats"][:, 1]) <= bl)
        assert np.all(np.abs(_np(ent) - o["entropy"]) <= be + 2 * u * o["entropy"]), (T, V)
        for got, want, bd in ((logp, o["logp"], bl), (tl, o["top_logp"], bl[:, None])):
            got, inf = _np(got), want == -np.inf
            assert np.array_equal(got == -np.inf, inf)
            with np.errstate(invalid="ignore"):
                assert np.all(inf | (np.abs(got - want) <= bd + 2 * u * np.abs(want))), (T, V)
        # the statistics alone, without tokens or alternatives
        stats2 = f(T, 2)
        km.kmp_token_logprobs(x, None, None, stats=stats2, workspace=ws)
        assert np.all(np.abs(_np(stats2).sum(axis=1) - o["lse"]) <= bl)
        # gradient at the statistics that were returned: p within (2|lp| + 8) u
        # and u times the sizes of the two subtractions' results, |lp| + log s
        g, h = rng.standard_normal(T), rng.standard_normal(T)
        gt, ht = (torch.as_tensor(v, device=device()).float() for v in (g, h))
        gv, hv, sv, Hv = _np(gt), _np(ht), _np(stats), _np(ent)
        with np.errstate(invalid="ignore"):
            lp = np.where(xv > -np.inf, (xv - sv[:, :1]) - sv[:, 1:], 0.0)
            p = np.where(xv > -np.inf, np.exp(lp), 0.0)
        term = p * (np.abs(gv)[:, None] + np.abs(hv)[:, None] * (np.abs(lp) + np.abs(Hv)[:, None]))
        bound = u * term * (4 * np.abs(lp) + 2 * np.abs(sv[:, 1:]) + 16) + 4 * u * np.abs(gv)[:, None] * (np.arange(V) == tok[:, None]) + 2.0 ** -120
        for use_h in (True, False):
            dx, _ = _put(np.zeros((T, V)), _dtype(xt), pad, off)
            km.kmp_token_logprobs_backward(x, tokens, stats, gt, dx, entropy=ent if use_h else None,
                                           dentropy=ht if use_h else None)
            want = OO.token_logprobs_backward(xv, tok, sv, gv, Hv, hv if use_h else None)
            assert np.all(np.abs(_np(dx) - want) <= bound + (uo if xt != "f32" else 0) * (np.abs(want) + bound) + TINY[xt]), (T, V)
        # in place
        km.kmp_token_logprobs_backward(x, tokens, stats, gt, x)
        assert torch.equal(x, dx)


def _edge_rows(V, lowest):
    """Rows that go wrong easily."""
    rng = np.random.default_rng(V)
    n = -np.inf
    rows = [np.full(V, n), np.full(V, 1.5), np.full(V, lowest), np.arange(V) % 100.0, -(np.arange(V) % 100.0)]
    few = np.full(V, n)
    few[[V - 1, V // 2, 3]] = 1.0, 2.0, 1.0         # three tokens allowed, at the far end
    rows.append(few)
    low = np.full(V, lowest)
    low[V // 3] = 0.0
    rows.append(low)
    r = rng.standard_normal(V)
    r[V // 2] = np.nan
    rows.append(r)
    r = rng.standard_normal(V)
    r[V // 4], r[5] = np.inf, n
    rows.append(r)
    rows.append(np.where(rng.random(V) < 0.5, 0.0, -0.0))        # equal zeros of both signs
    rows.append(np.sort(rng.standard_normal(V)))                 # the best ones last, in one place
    r = np.zeros(V)
    r[V - V // 3:] = 4.0                            # thousands of equal best ones
    rows.append(r)
    r = rng.standard_normal(V)
    r[0] = 3.0e4                                    # all probability in one token
    rows.append(r)
    return np.array(rows)


@pytest.mark.parametrize("xt", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("V", [70, 1000, 8191, 20011, 50000])
@pytest.mark.parametrize("copies", [1, 40])
def test_token_logprobs_rows_that_go_wrong_easily(xt, V, copies):
    """Few rows and many rows (which may take different forms)."""
    import torch
    from paper_2606_06742_amd import kmpath as km
    announce(f"token logprobs edges {xt} V {V} copies {copies}")
    lowest = {"f32": -3.4028234663852886e38, "bf16": -3.3895313892515355e38, "f16": -65504.0}[xt]
    base = _edge_rows(V, lowest)
    B = base.shape[0]
    one, onev = _put(base, _dtype(xt))
    x = one.repeat(copies, 1)
    T = B * copies
    tok = np.tile(np.array([1, V - 1, 2, V, 7, 3, V // 3, 1, V // 4, 0, V - 1, V - 1, 0])[:B], copies)
    tokens = torch.as_tensor(tok, device=device())
    f = lambda *s: torch.empty(*s, device=device())
    for top in (1, 20, 64):
        logp, ent, stats, tl, ti = f(T), f(T), f(T, 2), f(T, top), torch.empty(T, top, dtype=torch.int32, device=device())
        ws = torch.empty(km.kmp_token_logprobs_workspace_bytes(T, V, top), dtype=torch.uint8, device=device())
        ws.fill_(255)
        km.kmp_token_logprobs(x, tokens, logp, entropy=ent, stats=stats, top_id=ti, top_logp=tl, workspace=ws)
        o = OO.token_logprobs(onev, tok[:B], top)
        with np.errstate(all="ignore"):
            bl, be = _logprob_bounds(np.where(np.isfinite(onev), onev, np.where(np.isnan(onev), 0.0, onev)), o)
        # rows whose result is not finite, and one at the type's lowest value
        # (lse = lowest + log V rounds to a value of its own size)
        bl = np.where(np.isfinite(bl), bl, 0.0)
        be = np.where(np.isfinite(be), be, 0.0)
        assert np.array_equal(ti.cpu().numpy(), np.tile(o["top_id"], (copies, 1)))
        for got, want, bd in ((stats, o["stats"], bl[:, None]), (ent, o["entropy"], be), (logp, o["logp"], bl), (tl, o["top_logp"], bl[:, None])):
            got, want = _np(got), np.tile(want, (copies,) + (1,) * (want.ndim - 1))
            bd = np.tile(bd, (copies,) + (1,) * (bd.ndim - 1))
            same = (got == want) | (np.isnan(got) & np.isnan(want))
            with np.errstate(invalid="ignore"):
                ok = same | (np.abs(got - want) <= bd + 2 * U["f32"] * np.abs(want))
            assert np.all(ok), (top, np.argwhere(~ok)[:4], got[~ok][:4], want[~ok][:4])
    dx = torch.empty_like(x)
    g = torch.ones(T, device=device())
    km.kmp_token_logprobs_backward(x, tokens, stats, g, dx, entropy=ent, dentropy=g)
    want = OO.token_logprobs_backward(onev, tok[:B], _np(stats)[:B], np.ones(B), _np(ent)[:B], np.ones(B))
    want = np.tile(want, (copies, 1))
    got = _np(dx)
    assert np.array_equal(np.isnan(got), np.isnan(want))
    fin = np.isfinite(want)
    # p (1 + |log p| + H) <= 1 + log V + H: 1e-5 is 16 roundings of it and the type's
    assert np.all(np.abs(got[fin] - want[fin]) <= 1e-5 + U[xt] * np.abs(want[fin]))


def test_operators_replayed_from_a_graph():
    """Captured into a graph and replayed on new inputs, with eager work between
    the replays: the eager results every time."""
    import torch
    from paper_2606_06742_amd import kmpath as km
    announce("operators in a graph")
    dev = device()
    T, K, N, top = 3, 640, 4100, 5
    gen = torch.Generator(device="cuda")
    gen.manual_seed(5)
    x = torch.randn(T, K, generator=gen, device=dev).bfloat16()
    g, b = torch.ones(K, device=dev).bfloat16(), torch.zeros(K, device=dev).bfloat16()
    w = torch.randint(-127, 128, (N, K), generator=gen, device=dev, dtype=torch.int8)
    wscale = torch.full((N,), 1e-3, device=dev)
    tok = torch.tensor([1, 5, -1], device=dev)
    grad = torch.full((T,), -0.5, device=dev)

    def buffers():
        f = lambda *s: torch.zeros(*s, device=dev)
        return dict(q=torch.zeros(T, K, dtype=torch.int8, device=dev), s=f(T), y=torch.zeros_like(x), m=f(T), r=f(T),
                    l=f(T, N), lp=f(T), H=f(T), st=f(T, 2), ti=torch.zeros(T, top, dtype=torch.int32, device=dev),
                    tl=f(T, top), dl=f(T, N), dx=torch.zeros_like(x), dg=torch.zeros_like(g), db=torch.zeros_like(b),
                    ws=torch.zeros(km.kmp_token_logprobs_workspace_bytes(T, N, top), dtype=torch.uint8, device=dev),
                    wn=torch.zeros(km.kmp_layer_norm_workspace_bytes(T, K, torch.bfloat16), dtype=torch.uint8, device=dev))

    def work(v):
        km.kmp_layer_norm(x, g, b, EPS, v["q"], scale=v["s"])
        km.kmp_layer_norm(x, g, b, EPS, v["y"], mean=v["m"], rstd=v["r"])
        km.kmp_quantized_product(v["q"], v["s"], w, wscale, v["l"])
        km.kmp_token_logprobs(v["l"], tok, v["lp"], entropy=v["H"], stats=v["st"], top_id=v["ti"], top_logp=v["tl"],
                              workspace=v["ws"])
        km.kmp_token_logprobs_backward(v["l"], tok, v["st"], grad, v["dl"], entropy=v["H"], dentropy=grad)
        km.kmp_layer_norm_backward(v["y"], x, g, v["m"], v["r"], v["dx"], v["dg"], v["db"], v["wn"])

    eager, kept = buffers(), buffers()
    work(kept)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        work(kept)
    for i in range(4):
        x.copy_(torch.randn(T, K, generator=gen, device=dev))
        graph.replay()
        torch.cuda.synchronize()
        work(eager)
        torch.cuda.synchronize()
        for k in eager:
            if k not in ("ws", "wn"):
                assert torch.equal(eager[k], kept[k]), (i, k)


@pytest.mark.parametrize("xt", ["f32", "bf16", "f16"])
def test_token_logprobs_of_masks_alone(xt):
    """Rows and whole segments made of -inf and the type's lowest value: the
    alternatives by index among equals, probabilities shared by the lowest ones."""
    import torch
    from paper_2606_06742_amd import kmpath as km
    announce(f"token logprobs of masks alone {xt}")
    lowest = {"f32": -3.4028234663852886e38, "bf16": -3.3895313892515355e38, "f16": -65504.0}[xt]
    for V in (37, 9000, 70000):
        a = np.full((5, V), -np.inf)
        a[0, ::3] = lowest                        # both, mixed
        a[1, V // 2:] = lowest                    # segments of one or the other
        a[2, : V - 1] = lowest
        a[3, V - 1] = lowest                      # the only possible token
        a[4, : V // 2] = lowest
        a[4, V - 2] = 1.0
        x, xv = _put(a, _dtype(xt))
        tok = np.array([3, V - 1, V - 1, V - 1, 0])
        for top in (3, 20):
            f = lambda *s: torch.empty(*s, device=device())
            logp, ent, stats, tl, ti = f(5), f(5), f(5, 2), f(5, top), torch.empty(5, top, dtype=torch.int32, device=device())
            ws = torch.empty(km.kmp_token_logprobs_workspace_bytes(5, V, top), dtype=torch.uint8, device=device())
            km.kmp_token_logprobs(x, torch.as_tensor(tok, device=device()), logp, entropy=ent, stats=stats, top_id=ti,
                                  top_logp=tl, workspace=ws)
            o = OO.token_logprobs(xv, tok, top)
            assert np.array_equal(ti.cpu().numpy(), o["top_id"])
            # every term is exp(0) = 1 or 0: s is exact, log s within 2u of itself
            for got, want in ((logp, o["logp"]), (ent, o["entropy"]), (stats, o["stats"]), (tl, o["top_logp"])):
                got = _np(got)
                with np.errstate(invalid="ignore"):
                    assert np.all((got == want) | (np.abs(got - want) <= 4 * U["f32"] * np.abs(want))), (V, top)

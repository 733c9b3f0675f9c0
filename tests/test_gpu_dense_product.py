"""Products with bias, activation and residual, and their gradients, on the GPU against
oracle/operators.py (64 bits): types, sizes around every form's borders, strides,
unaligned rows, single tokens, missing operands, replays from a graph.

Bounds. u = 2^-24. A sum of K products is formed in chains of at most K/2 additions: it
is in error by at most (K/2 + 16) u times the sum of the products' sizes. The activations
have slopes of at most 1.13, and their own evaluation is taken to be within 16 u (1 + |z|
+ z^2). Rounding to the output's type adds uo of the result."""
import numpy as np
import pytest

from oracle import operators as OO
from tests.gpu_common import announce, device
from tests.test_gpu_operators import TINY, U, _dtype, _np, _put

pytestmark = pytest.mark.gpu

u = U["f32"]
ACTS = ["none", "relu", "gelu", "gelu_tanh", "silu"]
# M, N, K: single tokens, odd sizes, the forms' borders
SIZES = [(1, 1, 1), (1, 64, 64), (3, 7, 5), (1, 4096, 1000), (5, 1003, 333), (16, 256, 512), (17, 65, 129), (33, 100, 1), (64, 64, 128),
         (40, 3001, 257), (100, 130, 2050), (200, 1999, 77), (257, 255, 640), (300, 700, 1030)]


def _vec(a, dtype):
    t, v = _put(a[None], dtype)
    return t[0], v[0]


def _inputs(rng, M, N, K, xt, pad=0, off=0, scale=1.0):
    x = _put(rng.standard_normal((M, K)) * np.exp(0.3 * rng.standard_normal(K)) + 0.1, _dtype(xt), pad, off)
    w = _put(scale * rng.standard_normal((N, K)) / np.sqrt(max(K, 1)), _dtype(xt), pad, off)
    return x, w


def _close(got, want, bound, t):
    uo = U[t] if t != "f32" else u
    return np.all(np.abs(_np(got) - want) <= bound + uo * (np.abs(want) + bound) + TINY[t])


def _check_forward(rng, M, N, K, xt, ot, bt, act, residual, keep, pad, off):
    import torch
    from paper_2606_06742_amd import kmpath as km
    (x, xv), (w, wv) = _inputs(rng, M, N, K, xt, pad, off)
    b, bv = (None, None) if bt is None else _vec(0.3 * rng.standard_normal(N), _dtype(bt))
    r, rv = (None, None) if not residual else _put(rng.standard_normal((M, N)), _dtype(ot), pad, off)
    out = _put(np.zeros((M, N)), _dtype(ot), pad, off)[0]
    z = _put(np.zeros((M, N)), _dtype(xt), pad, off)[0] if keep else None
    km.kmp_dense_product(x, w, out, bias=b, act=act, residual=r, z=z)
    oe, ze = OO.dense_product(xv, wv, bv, act, rv)
    size = np.abs(xv) @ np.abs(wv).T
    ez = (K / 2 + 16) * u * size + 2 * u * (np.abs(ze) + (0 if bv is None else np.abs(bv)))
    eo = 1.13 * ez + (0 if act == "none" else 16 * u * (1 + np.abs(ze) + ze * ze)) + 2 * u * (0 if rv is None else np.abs(rv))
    assert _close(out, oe, eo, ot), np.abs(_np(out) - oe).max()
    assert z is None or _close(z, ze, ez, xt)
    return x, w, out, oe


@pytest.mark.parametrize("xt,ot", [("f32", "f32"), ("bf16", "bf16"), ("bf16", "f32"), ("f16", "f16"), ("f16", "f32")])
def test_forward(xt, ot):
    for i, (M, N, K) in enumerate(SIZES):
        for j, (pad, off) in enumerate(((0, 0), (1, 1))):
            act, bt = ACTS[(i + j) % 5], (None, xt, "f32")[(i + 2 * j) % 3]
            residual, keep = (i + j) % 2 == 0, (i + j) % 3 == 0
            announce(f"dense product {xt} to {ot} {M} x {N} x {K} gap {pad} {act} bias {bt} residual {residual} z {keep}")
            _check_forward(np.random.default_rng(100 * i + j), M, N, K, xt, ot, bt, act, residual, keep, pad, off)


@pytest.mark.parametrize("xt", ["f32", "bf16", "f16"])
def test_forward_of_large_tiles(xt):
    """Sizes that take every larger form, aligned and not, K with and without a rest."""
    for M, N, K, pad in ((1025, 1030, 128, 0), (700, 5000, 200, 0), (4097, 3100, 64, 0), (1500, 1500, 333, 0), (2500, 1900, 160, 8),
                         (3500, 3700, 200, 1), (129, 8200, 1031, 1), (16, 20000, 256, 0), (64, 9000, 256, 0)):
        announce(f"dense product {xt} {M} x {N} x {K} gap {pad}")
        _check_forward(np.random.default_rng(M + N), M, N, K, xt, xt, "f32", "gelu", True, True, pad, 0)


@pytest.mark.parametrize("xt", ["f32", "bf16", "f16"])
def test_every_place_once(xt):
    """x and w of one 1 a row each: every product is 0 or 1, exactly; any wrong index shows."""
    import torch
    from paper_2606_06742_amd import kmpath as km
    for M, N, K in ((33, 65, 70), (300, 500, 96), (1000, 2000, 129), (2100, 8400, 72), (1200, 1300, 1048), (40, 2500, 2056)):
        announce(f"dense product, ones, {xt} {M} x {N} x {K}")
        rng = np.random.default_rng(M)
        i, j = torch.as_tensor(rng.integers(0, K, M), device=device()), torch.as_tensor(rng.integers(0, K, N), device=device())
        x, w = torch.zeros(M, K, dtype=_dtype(xt), device=device()), torch.zeros(N, K, dtype=_dtype(xt), device=device())
        x[torch.arange(M, device=device()), i] = 1
        w[torch.arange(N, device=device()), j] = 1
        out = torch.empty(M, N, dtype=_dtype(xt), device=device())
        km.kmp_dense_product(x, w, out)
        assert torch.equal(out, (i[:, None] == j[None, :]).to(out.dtype))
        # gradients of the same kind: dx of one 1 per row of dout, dw likewise
        dx, dw = torch.empty_like(x), torch.empty_like(w)
        ws = torch.full((km.kmp_dense_product_workspace_bytes(M, N, K, x.dtype),), 255, dtype=torch.uint8, device=device())
        at = torch.as_tensor(rng.integers(0, N, M), device=device())
        dout = torch.zeros_like(out)
        dout[torch.arange(M, device=device()), at] = 1
        db = torch.empty(N, device=device())
        km.kmp_dense_product_backward(dout, x, w, None, dx, dw, db, workspace=ws)
        assert torch.equal(dx, w[at])
        want = torch.zeros(N, K, device=device()).index_add_(0, at, x.float())
        assert torch.equal(dw.float(), want) and torch.equal(db, want.sum(dim=1))


def test_precision():
    """The error of 32-bit products, and of 16-bit ones with 32-bit outputs, in the mean:
    random roundings of chains of K/2 additions are within sqrt(K) u of the result."""
    from paper_2606_06742_amd import kmpath as km
    import torch
    for xt, M, N, K in (("f32", 200, 300, 2000), ("bf16", 200, 300, 4000), ("f16", 1200, 900, 1000), ("bf16", 1, 3000, 3000)):
        announce(f"dense product, precision {xt} {M} x {N} x {K}")
        rng = np.random.default_rng(K)
        (x, xv), (w, wv) = _inputs(rng, M, N, K, xt)
        out = torch.empty(M, N, device=device())
        km.kmp_dense_product(x, w, out)
        e = xv @ wv.T
        assert np.linalg.norm(_np(out) - e) <= np.sqrt(K) * u * np.linalg.norm(e)


def _check_backward(rng, M, N, K, xt, act, pad, off, bt="f32"):
    import torch
    from paper_2606_06742_amd import kmpath as km
    (x, xv), (w, wv) = _inputs(rng, M, N, K, xt, pad, off)
    z, zv = _put(1.5 * rng.standard_normal((M, N)), _dtype(xt), pad, off)
    do, dov = _put(rng.standard_normal((M, N)) + 0.1, _dtype(xt), pad, off)
    dx, dw = (_put(np.zeros(s), _dtype(xt), pad, off)[0] for s in ((M, K), (N, K)))
    db = torch.empty(N, dtype=_dtype(bt), device=device())
    need = km.kmp_dense_product_workspace_bytes(M, N, K, _dtype(xt))
    ws = torch.full((need,), 255, dtype=torch.uint8, device=device())
    km.kmp_dense_product_backward(do, x, w, None if act == "none" else z, dx, dw, db, act=act, workspace=ws)
    dxe, dwe, dbe, dz = OO.dense_product_backward(dov, xv, wv, zv, act)
    # dz: the slope within 16 u (1 + |z| + z^2), then its rounding to the type of the products
    es = 0 if act == "none" else np.abs(dov) * 16 * u * (1 + np.abs(zv) + zv * zv) + 2 * u * np.abs(dz)
    er = es if act == "none" or xt == "f32" else es + U[xt] * (np.abs(dz) + es) + TINY[xt]
    az = np.abs(dz)
    ex = er @ np.abs(wv) if act != "none" else 0
    ex = ex + (N / 2 + 16) * u * (az @ np.abs(wv))
    ew = er.T @ np.abs(xv) if act != "none" else 0
    ew = ew + (M / 2 + 16) * u * (az.T @ np.abs(xv))
    eb = (0 if act == "none" else es.sum(axis=0)) + (M / 2 + 16) * u * az.sum(axis=0)
    assert _close(dx, dxe, ex, xt), np.abs(_np(dx) - dxe).max()
    assert _close(dw, dwe, ew, xt), np.abs(_np(dw) - dwe).max()
    assert _close(db, dbe, eb, bt), np.abs(_np(db) - dbe).max()
    # the same again, and each alone
    dx2, dw2, db2 = torch.empty_like(dx), torch.empty_like(dw), torch.empty_like(db)
    zz = None if act == "none" else z
    km.kmp_dense_product_backward(do, None, w, zz, dx2, None, None, act=act, workspace=ws)
    km.kmp_dense_product_backward(do, x, None, zz, None, dw2, None, act=act, workspace=ws)
    km.kmp_dense_product_backward(do, None, None, zz, None, None, db2, act=act, workspace=ws)
    assert torch.equal(dx, dx2) and torch.equal(dw, dw2) and torch.equal(db, db2)


@pytest.mark.parametrize("xt", ["f32", "bf16", "f16"])
def test_backward(xt):
    for i, (M, N, K) in enumerate(SIZES):
        for j, (pad, off) in enumerate(((0, 0), (1, 1))):
            act = ACTS[(i + 2 * j) % 5]
            announce(f"dense product backward {xt} {M} x {N} x {K} gap {pad} {act}")
            _check_backward(np.random.default_rng(100 * i + j), M, N, K, xt, act, pad, off, "f32" if j else xt)


@pytest.mark.parametrize("xt", ["f32", "bf16", "f16"])
def test_backward_of_large_tiles(xt):
    for M, N, K, pad, act in ((1100, 1300, 700, 0, "gelu"), (2600, 500, 1900, 1, "silu"), (130, 4200, 2100, 0, "relu"),
                              (8, 4096, 1500, 0, "gelu_tanh"), (2, 1500, 5000, 1, "gelu")):
        announce(f"dense product backward {xt} {M} x {N} x {K} gap {pad} {act}")
        _check_backward(np.random.default_rng(M + N), M, N, K, xt, act, pad, 0)


@pytest.mark.parametrize("xt", ["bf16", "f16"])
def test_backward_of_operands_as_they_are(xt):
    """Rows of whole 16 bytes, at multiples of them: w and x are not transposed first. Depths
    with and without a rest, fewer than a slice, columns that end inside a tile, channels
    that are no multiple of 8; and rows just not aligned beside them."""
    for M, N, K, pad, act in ((700, 1003, 1104, 0, "gelu"), (300, 2051, 1024, 8, "silu"), (2100, 1500, 2304, 0, "none"),
                              (60, 1030, 8200, 16, "relu"), (1025, 17, 1032, 0, "gelu"), (4100, 3000, 520, 0, "gelu_tanh"),
                              (700, 1003, 1104, 4, "gelu")):
        announce(f"dense product backward, operands as they are, {xt} {M} x {N} x {K} gap {pad} {act}")
        _check_backward(np.random.default_rng(M + N), M, N, K, xt, act, pad, 0)


def test_relu_at_zero_and_extreme_values():
    """act'(0) = 0 for relu; the activations and slopes at large |z|, of NaN and infinities."""
    import torch
    from paper_2606_06742_amd import kmpath as km
    z = np.array([[0.0, -0.0, 1e-30, -1e-30, 90.0, -90.0, 1e4, -1e4, 3e38, -3e38, 2.0, -2.0]])
    x = torch.as_tensor(z.T.copy(), device=device()).float()           # z as products with 1
    one = torch.ones(1, 1, device=device())
    dout = torch.ones(len(x), 1, device=device())
    for act in ACTS:
        announce(f"dense product, extreme values, {act}")
        out, zo = torch.empty(len(x), 1, device=device()), torch.empty(len(x), 1, device=device())
        km.kmp_dense_product(x, one, out, act=act, z=zo)
        assert torch.equal(zo, x)
        zs = x.double().cpu().numpy()
        with np.errstate(over="ignore", invalid="ignore"):
            a, d = OO.activation(np.clip(zs, -1e30, 1e30), act)
        a = np.where(np.abs(zs) > 1e30, np.where(zs > 0, zs, zs if act == "none" else 0.0), a)
        assert np.all(np.abs(_np(out) - a) <= 16 * u * (1 + np.minimum(np.abs(zs), 10.0)) + 2 * u * np.abs(a)), (act, _np(out), a)
        dx = torch.empty_like(x)
        ws = torch.empty(km.kmp_dense_product_workspace_bytes(len(x), 1, 1, x.dtype), dtype=torch.uint8, device=device())
        km.kmp_dense_product_backward(dout, None, one, zo, dx, None, None, act=act, workspace=ws)
        d = np.where(np.abs(zs) > 1e3, np.where((zs > 0) | (act == "none"), 1.0, 0.0), d)
        assert np.all(np.abs(_np(dx) - d) <= 64 * u), (act, _np(dx), d)
        x2 = torch.tensor([[float("nan")], [1.0]], device=device())
        out = torch.empty(2, 1, device=device())
        km.kmp_dense_product(x2, one, out, act=act)
        assert bool(out[0].isnan().all()) and not bool(out[1].isnan().any())


def test_empty_sizes_and_in_place():
    """No tokens, channels or depth; out written over the residual."""
    import torch
    from paper_2606_06742_amd import kmpath as km
    for dtype in (torch.float32, torch.bfloat16):
        e = lambda *s: torch.full(s, 3.0, dtype=dtype, device=device())
        ws = torch.empty(1 << 20, dtype=torch.uint8, device=device())
        out, bias, res = e(5, 6), torch.arange(6.0, device=device()), e(5, 6)
        km.kmp_dense_product(e(5, 0), e(6, 0), out, bias=bias, act="relu", residual=res)
        assert torch.equal(out.float(), (bias + 3.0).expand(5, 6))
        km.kmp_dense_product(e(0, 4), e(6, 4), e(0, 6))
        km.kmp_dense_product(e(5, 4), e(0, 4), e(5, 0))
        dx, dw, db = e(5, 4), e(6, 4), torch.full((6,), 3.0, device=device())
        km.kmp_dense_product_backward(e(0, 6), e(0, 4), e(6, 4), None, e(0, 4), dw, db, workspace=ws)
        assert bool((dw == 0).all()) and bool((db == 0).all())
        km.kmp_dense_product_backward(e(5, 0), e(5, 4), e(0, 4), None, dx, e(0, 4), e(0).float(), workspace=ws)
        assert bool((dx == 0).all())
        km.kmp_dense_product_backward(e(5, 6), e(5, 0), e(6, 0), None, e(5, 0), e(6, 0), db, workspace=ws)
        assert bool((db == 15).all())
        x, w = torch.randn(70, 50, device=device()).to(dtype), torch.randn(90, 50, device=device()).to(dtype)
        res = torch.randn(70, 90, device=device()).to(dtype)
        out = torch.empty_like(res)
        km.kmp_dense_product(x, w, out, act="silu", residual=res)
        km.kmp_dense_product(x, w, res, act="silu", residual=res)
        assert torch.equal(out, res)


def test_replayed_from_a_graph():
    import torch
    from paper_2606_06742_amd import kmpath as km
    for M in (1, 200):
        N, K = 700, 512
        g0 = torch.Generator(device=device())
        g0.manual_seed(M)
        r = lambda *s: torch.randn(*s, generator=g0, device=device()).to(torch.bfloat16)
        x, w, b, do = r(M, K), r(N, K), r(N), r(M, N)
        ws = torch.empty(km.kmp_dense_product_workspace_bytes(M, N, K, x.dtype), dtype=torch.uint8, device=device())

        def step():
            o = [torch.empty(M, N, dtype=x.dtype, device=device()) for _ in range(2)] + [torch.empty_like(x), torch.empty_like(w),
                                                                                         torch.empty_like(b)]
            km.kmp_dense_product(x, w, o[0], bias=b, act="gelu", z=o[1])
            km.kmp_dense_product_backward(do, x, w, o[1], o[2], o[3], o[4], act="gelu", workspace=ws)
            return o

        step()
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            out = step()
        for i in range(4):
            announce(f"dense product replay {i} of {M} tokens")
            x.mul_(0.9)
            do.add_(0.1)
            g.replay()
            torch.cuda.synchronize()
            got = [t.clone() for t in out]
            assert all(torch.equal(p, q) for p, q in zip(got, step()))


def test_gradients_against_differences():
    """Differences of the library's own outputs in 32 bits along random directions, steps
    of 2^-7 either way: within 2 % of the gradient's size (third derivatives of the order
    1 over 10^4, rounding of 2^-24 of the loss over 2^-7)."""
    import torch
    from paper_2606_06742_amd import kmpath as km
    M, N, K = 9, 14, 21
    g0 = torch.Generator(device=device())
    g0.manual_seed(1)
    r = lambda *s: torch.randn(*s, generator=g0, device=device())
    for act in ("none", "gelu", "gelu_tanh", "silu"):
        x, w, b, c = r(M, K), r(N, K) / K ** 0.5, r(N), r(M, N)
        out, z = torch.empty(M, N, device=device()), torch.empty(M, N, device=device())

        def loss():
            km.kmp_dense_product(x, w, out, bias=b, act=act, z=z)
            return float((out.double() * c.double()).sum())

        loss()
        grads = dx, dw, db = torch.empty_like(x), torch.empty_like(w), torch.empty_like(b)
        ws = torch.empty(km.kmp_dense_product_workspace_bytes(M, N, K, x.dtype), dtype=torch.uint8, device=device())
        km.kmp_dense_product_backward(c, x, w, z, dx, dw, db, act=act, workspace=ws)
        for t, g in zip((x, w, b), grads):
            step, keep = r(*t.shape), t.clone()
            t.copy_(keep + step / 128)
            up = loss()
            t.copy_(keep - step / 128)
            down = loss()
            t.copy_(keep)
            size = float((g.double() * step.double()).square().sum().sqrt())
            assert abs((up - down) * 64 - float((g.double() * step.double()).sum())) <= 2e-2 * size + 1e-3, act

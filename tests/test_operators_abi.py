"""The operators' entry points on the host: what they refuse before touching a
device, their workspace sizes, and the binding's checks of tensors."""
import os

import pytest
import torch

P = 0x1000        # stands in for a device pointer in calls that are refused


@pytest.fixture(scope="module")
def km():
    from paper_2606_06742_amd import kmpath
    if not os.path.exists(kmpath.LIB_PATH):
        from paper_2606_06742_amd import build
        build.build()
    kmpath.lib()
    return kmpath


def _norm(km, xt=1, x=P, rows=4, d=8, ldx=8, wt=1, g=P, b=P, eps=1e-5, yt=1, y=P, ldy=8, scale=None):
    return km.lib().kmp_layer_norm(None, xt, x, rows, d, ldx, wt, g, b, eps, yt, y, ldy, None, None, scale)


def test_layer_norm_refusals(km):
    bad = [dict(xt=4), dict(xt=-1), dict(xt=1, wt=2, g=P), dict(xt=0, wt=1), dict(yt=2), dict(xt=0, wt=0, yt=4, scale=P),
           dict(rows=-1), dict(d=0), dict(ldx=7), dict(ldy=7), dict(eps=-1e-9), dict(eps=float("nan")),
           dict(eps=float("inf")), dict(x=None), dict(y=None), dict(yt=4), dict(rows=1 << 40), dict(d=1 << 40, ldx=1 << 41)]
    for b in bad:
        assert _norm(km, **b) == km.KMP_EINVAL, b
        assert "kmp_layer_norm" in km.kmp_strerror(km.KMP_EINVAL)
    assert _norm(km, rows=0, x=None, y=None) == km.KMP_OK


def test_layer_norm_backward_refusals(km):
    L = km.lib()
    need = km.kmp_layer_norm_workspace_bytes(100, 8, torch.float32)

    def call(xt=1, dy=P, lddy=8, x=P, ldx=8, rows=100, d=8, wt=1, mean=P, rstd=P, dx=P, lddx=8, dg=P, db=P, ws=P, n=need):
        return L.kmp_layer_norm_backward(None, xt, dy, lddy, x, ldx, rows, d, wt, P, mean, rstd, dx, lddx, dg, db, ws, n)

    for b in (dict(xt=9), dict(wt=3), dict(lddy=7), dict(ldx=1), dict(lddx=7), dict(rows=-2), dict(d=0), dict(dy=None),
              dict(x=None), dict(mean=None), dict(rstd=None)):
        assert call(**b) == km.KMP_EINVAL, b
    assert call(ws=None) == km.KMP_EWORKSPACE and call(n=need - 1) == km.KMP_EWORKSPACE
    assert call(ws=P + 4) == km.KMP_EWORKSPACE
    assert call(dx=None, dg=None, db=None, ws=None) == km.KMP_OK       # nothing asked for
    assert L.kmp_layer_norm_workspace_bytes(7, 1, 1) == 0 and L.kmp_layer_norm_workspace_bytes(1, -1, 1) == 0


def test_quantized_refusals(km):
    L = km.lib()
    assert L.kmp_quantize_rows(None, 0, P, 1, 1, 1, P, 1, P) == km.KMP_EINVAL
    assert L.kmp_quantize_rows(None, 1, P, 1, 5, 4, P, 5, P) == km.KMP_EINVAL
    assert L.kmp_quantize_rows(None, 1, P, 1, 5, 5, P, 4, P) == km.KMP_EINVAL
    assert L.kmp_quantize_rows(None, 1, P, 1, 5, 5, P, 5, None) == km.KMP_EINVAL
    assert L.kmp_quantize_rows(None, 1, None, 0, 5, 5, None, 5, None) == km.KMP_OK

    def call(x=P, ldx=8, xs=P, M=2, w=P, ldw=8, ws=P, N=3, K=8, ot=1, out=P, ldo=3):
        return L.kmp_quantized_product(None, x, ldx, xs, M, w, ldw, ws, N, K, None, ot, out, ldo)

    for b in (dict(ot=0), dict(ot=4), dict(M=-1), dict(N=-1), dict(K=-1), dict(ldx=7), dict(ldw=7), dict(ldo=2),
              dict(x=None), dict(w=None), dict(xs=None), dict(ws=None), dict(out=None),
              dict(K=131072, ldx=131072, ldw=131072), dict(M=1 << 30, N=1 << 20, ldo=1 << 20)):
        assert call(**b) == km.KMP_EINVAL, b
    assert call(M=0, x=None) == km.KMP_OK and call(N=0, w=None, ldo=0) == km.KMP_OK


def test_token_logprobs_refusals(km):
    L = km.lib()
    need = km.kmp_token_logprobs_workspace_bytes(4, 100, 5)
    assert need > 0
    for T, V, top in ((-1, 5, 0), (1, 0, 0), (1, 5, 6), (1, 500, 65), (1, 5, -1)):
        assert km.kmp_token_logprobs_workspace_bytes(T, V, top) == 0

    def fwd(t=1, x=P, T=4, V=100, ld=100, bits=64, tok=P, lp=P, top=5, ws=P, n=need):
        return L.kmp_token_logprobs(None, t, x, T, V, ld, bits, tok, lp, None, None, top, P, P, ws, n)

    for b in (dict(t=0), dict(t=4), dict(x=None), dict(T=-1), dict(V=0), dict(ld=99), dict(bits=16), dict(tok=None),
              dict(top=101), dict(top=65), dict(top=-1)):
        assert fwd(**b) == km.KMP_EINVAL, b
    assert fwd(ws=None) == km.KMP_EWORKSPACE and fwd(n=need - 1) == km.KMP_EWORKSPACE
    assert fwd(ws=P + 8) == km.KMP_EWORKSPACE
    assert fwd(T=0, x=None, ws=None) == km.KMP_OK

    def bwd(t=1, x=P, T=4, V=100, ld=100, bits=32, tok=P, st=P, H=P, g=P, h=P, dx=P, ldd=100):
        return L.kmp_token_logprobs_backward(None, t, x, T, V, ld, bits, tok, st, H, g, h, dx, ldd)

    for b in (dict(t=0), dict(x=None), dict(T=-1), dict(V=0), dict(ld=99), dict(ldd=99), dict(bits=8), dict(tok=None),
              dict(st=None), dict(H=None), dict(dx=None)):
        assert bwd(**b) == km.KMP_EINVAL, b
    assert bwd(T=0, x=None) == km.KMP_OK


def test_binding_refuses_tensors(km):
    """Wrong place, shape, type, stride: refused with the argument's name."""
    x = torch.zeros(2, 3)
    with pytest.raises(km.KmpError, match="x must be a 2-D device tensor"):
        km.kmp_layer_norm(x, None, None, 1e-5, x)
    with pytest.raises(km.KmpError, match="logits"):
        km.kmp_token_logprobs(x, None, None)
    with pytest.raises(km.KmpError, match="xq"):
        km.kmp_quantized_product(x, None, x, None, x)

    class Fake:                                   # a device tensor's metadata
        def __init__(self, shape, stride, dtype=torch.float32):
            self.shape, self._s, self.dtype, self.is_cuda = shape, stride, dtype, True

        def dim(self):
            return len(self.shape)

        def stride(self):
            return self._s

        def numel(self):
            return self.shape[0]

        def is_contiguous(self):
            return self._s == (1,)

        def is_floating_point(self):
            return self.dtype.is_floating_point

        def element_size(self):
            return self.dtype.itemsize

        def data_ptr(self):
            return P

    assert km._matrix(Fake((4, 3), (5, 1)), "x") == (P, 4, 3, 5)
    assert km._matrix(Fake((1, 3), (1, 1)), "x") == (P, 1, 3, 3)      # one row: its stride means nothing
    for f in (Fake((4, 3), (1, 4)), Fake((4, 3), (2, 1)), Fake((4, 3), (3, 2)), Fake((4,), (1,)), Fake((4, 3), (0, 1))):
        with pytest.raises(km.KmpError):
            km._matrix(f, "x")
    with pytest.raises(km.KmpError):
        km._matrix(Fake((4, 3), (3, 1)), "y", 4, 5)
    with pytest.raises(km.KmpError):
        km._vector(Fake((4,), (2,)), "gamma", 4)
    with pytest.raises(km.KmpError):
        km._vector(Fake((4,), (1,)), "mean", 4, torch.float64)
    for dt in (torch.float32, torch.int16):
        with pytest.raises(km.KmpError):
            km._tokens(Fake((4,), (1,), dt), 4)
    with pytest.raises(km.KmpError):
        km._type(torch.complex64, "x")

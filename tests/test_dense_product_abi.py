"""kmp_dense_product on the host: refusals, workspace sizes, the binding's checks, and
the oracle's gradients against differences."""
import numpy as np
import pytest
import torch

from oracle import operators as OO
from tests.test_operators_abi import P, km  # noqa: F401


def test_forward_refusals(km):  # noqa: F811
    def call(t=2, x=P, ldx=8, M=4, w=P, ldw=8, N=6, K=8, bt=2, b=P, act=2, ot=2, res=P, ldr=6, out=P + 64, ldo=6, z=P, ldz=6):
        return km.lib().kmp_dense_product(None, t, x, ldx, M, w, ldw, N, K, bt, b, act, ot, res, ldr, out, ldo, z, ldz)

    for b in (dict(t=0, bt=0, ot=0), dict(t=4, bt=4, ot=4), dict(bt=3), dict(ot=3), dict(t=1, bt=2, ot=1), dict(act=-1), dict(act=5),
              dict(M=-1), dict(N=-1), dict(K=-1), dict(M=1 << 31), dict(K=(1 << 28) + 1, ldx=1 << 29, ldw=1 << 29), dict(ldx=7),
              dict(ldw=7), dict(ldo=5), dict(ldr=5), dict(ldz=5), dict(ldo=(1 << 40) + 1), dict(x=None), dict(w=None), dict(out=None),
              dict(out=P, ldo=7), dict(M=1 << 30, N=1 << 20, ldo=1 << 20, ldr=1 << 20, ldz=1 << 20)):
        assert call(**b) == km.KMP_EINVAL, b
        assert "kmp_dense_product" in km.kmp_strerror(km.KMP_EINVAL)
    assert call(M=0, x=None, out=None) == km.KMP_OK and call(N=0, w=None, out=None, ldo=0) == km.KMP_OK


def test_backward_refusals(km):  # noqa: F811
    need = km.kmp_dense_product_workspace_bytes(4, 6, 8, torch.bfloat16)

    def call(t=2, do=P, lddo=6, M=4, N=6, K=8, act=2, z=P, ldz=6, x=P, ldx=8, w=P, ldw=8, dx=P, lddx=8, dw=P, lddw=8, bt=2, db=P,
             ws=P, n=need):
        return km.lib().kmp_dense_product_backward(None, t, do, lddo, M, N, K, act, z, ldz, x, ldx, w, ldw, dx, lddx, dw, lddw, bt, db,
                                                   ws, n)

    for b in (dict(t=0), dict(bt=3), dict(act=5), dict(M=-1), dict(N=-1), dict(K=-1), dict(M=(1 << 28) + 1), dict(lddo=5), dict(ldz=5),
              dict(ldx=7), dict(ldw=7), dict(lddx=7), dict(lddw=7), dict(do=None), dict(z=None), dict(x=None), dict(w=None),
              dict(M=1 << 28, N=1 << 20, lddo=1 << 20, ldz=1 << 20), dict(N=1 << 28, K=1 << 12, lddo=1 << 28, ldz=1 << 28, ldx=1 << 12,
                                                                         ldw=1 << 12, lddx=1 << 12, lddw=1 << 12)):
        assert call(**b) == km.KMP_EINVAL, b
    assert call(ws=None) == km.KMP_EWORKSPACE and call(n=need - 1) == km.KMP_EWORKSPACE and call(ws=P + 4) == km.KMP_EWORKSPACE
    assert call(dx=None, dw=None, db=None, ws=None) == km.KMP_OK        # nothing asked for
    size = km.lib().kmp_dense_product_workspace_bytes
    for a in ((0, 1, 1, 1), (4, 1, 1, 1), (1, -1, 1, 1), (1, 1, -1, 1), (1, 1, 1, -1), (1, 1, 1, (1 << 28) + 1)):
        assert size(*a) == 0
    assert size(1, 0, 0, 0) >= 256


def test_workspace_does_not_fall(km):  # noqa: F811
    """A workspace of a program's largest call serves its smaller ones."""
    some = [0, 1, 2, 4, 7, 8, 15, 16, 17, 31, 32, 33, 63, 64, 65, 100, 127, 128, 129, 200, 255, 256, 257, 1000, 4096, 4097, 20000]
    size = km.lib().kmp_dense_product_workspace_bytes
    for t in (1, 2, 3):
        for a in (1, 9, 64, 1000, 4096):
            for b in (1, 65, 2048):
                for order in ((0, 1, 2), (1, 0, 2), (1, 2, 0)):
                    sizes = [size(t, *[(v, a, b)[i] for i in order]) for v in some]
                    assert sizes == sorted(sizes), (t, a, b, order)


def test_binding_refuses(km):  # noqa: F811
    x = torch.zeros(2, 3)
    with pytest.raises(km.KmpError, match="x must be a 2-D device tensor"):
        km.kmp_dense_product(x, x, x)
    with pytest.raises(km.KmpError, match="dout must be a 2-D device tensor"):
        km.kmp_dense_product_backward(x, x, x, x, None, None, None)
    with pytest.raises(km.KmpError, match="activation 'tanh' is not one of none, relu"):
        km._act("tanh")
    assert [km._act(a) for a in ("none", "relu", "gelu", "gelu_tanh", "silu")] == [0, 1, 2, 3, 4]


@pytest.mark.parametrize("act", ["none", "relu", "gelu", "gelu_tanh", "silu"])
def test_oracle_gradients_against_differences(act):
    """Central differences in 64 bits, step 1e-6, away from relu's border."""
    rng = np.random.default_rng(1)
    x, w, b, c = (rng.standard_normal(s) for s in ((4, 5), (6, 5), (6,), (4, 6)))
    _, z = OO.dense_product(x, w, b, act)
    assert np.abs(z).min() > 1e-3
    dx, dw, db, _ = OO.dense_product_backward(c, x, w, z, act)
    loss = lambda x, w, b: (OO.dense_product(x, w, b, act)[0] * c).sum()
    for k, (p, g) in enumerate(((x, dx), (w, dw), (b, db))):
        for i in np.ndindex(p.shape):
            step = np.zeros_like(p)
            step[i] = 1e-6
            args = [[x, w, b], [x, w, b]]
            args[0][k], args[1][k] = p + step, p - step
            assert abs((loss(*args[0]) - loss(*args[1])) / 2e-6 - g[i]) <= 1e-6 * (1 + abs(g[i]))


def test_largest_arguments(km):  # noqa: F811
    """Workspaces of the largest accepted sizes do not overflow."""
    most = 1 << 28
    size = km.lib().kmp_dense_product_workspace_bytes
    for t in (1, 2, 3):
        for m, n, k in ((most, most, most), (most, 1, 1), (1, most, 1), (1, 1, most), (16, most, most), (0, most, most)):
            assert 256 <= size(t, m, n, k) < 1 << 62

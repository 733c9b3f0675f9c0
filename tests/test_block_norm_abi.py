"""kmp_block_norm on the host: what it refuses before touching a device, its workspace
sizes, the binding's checks, and the oracle's gradients against differences."""
import numpy as np
import pytest
import torch

from oracle import operators as OO
from tests.test_operators_abi import P, km  # noqa: F401


def test_forward_refusals(km):  # noqa: F811
    def call(xt=2, flags=2, b=P, ldb=8, res=P, ldr=8, rows=4, d=8, wt=2, gate=P, ldg=0, rscale=1.0, eps=1e-5, h=P + 64, ldh=8,
             yt=2, y=P, ldy=8, scale=None):
        return km.lib().kmp_block_norm(None, xt, flags, b, ldb, res, ldr, rows, d, wt, P, P, gate, ldg, rscale, P, P, eps, h, ldh,
                                       yt, y, ldy, None, scale)

    bad = [dict(xt=0, wt=0, yt=0), dict(xt=4), dict(wt=3), dict(xt=1, wt=2, yt=1), dict(flags=4), dict(flags=-1), dict(yt=1),
           dict(yt=4), dict(rows=-1), dict(rows=1 << 31), dict(d=0), dict(ldb=7), dict(ldr=7), dict(ldh=7), dict(ldy=7),
           dict(ldg=7), dict(ldg=-1), dict(ldb=(1 << 40) + 1), dict(eps=-1.0), dict(eps=float("nan")), dict(rscale=float("inf")),
           dict(h=None, y=None), dict(h=P, ldh=9), dict(b=None)]
    for b in bad:
        assert call(**b) == km.KMP_EINVAL, b
        assert "kmp_block_norm" in km.kmp_strerror(km.KMP_EINVAL)
    assert call(rows=0, b=None, res=None, h=None, y=None) == km.KMP_OK


def test_backward_refusals(km):  # noqa: F811
    need = km.kmp_block_norm_workspace_bytes(100, 8, torch.bfloat16)

    def call(xt=2, flags=2, dy=P, lddy=8, dh=P, lddh=8, b=P, ldb=8, h=P, ldh=8, rows=100, d=8, wt=2, gate=P, ldg=0, rscale=1.0,
             st=P, db=P, lddb=8, dres=P, lddr=8, dgate=P, lddg=0, dga=P, dba=P, dg=P, dbe=P, ws=P, n=need):
        return km.lib().kmp_block_norm_backward(None, xt, flags, dy, lddy, dh, lddh, b, ldb, h, ldh, rows, d, wt, P, P, gate, ldg,
                                                rscale, P, st, db, lddb, dres, lddr, dgate, lddg, dga, dba, dg, dbe, ws, n)

    for b in (dict(xt=0), dict(wt=3), dict(flags=8), dict(lddy=7), dict(lddh=7), dict(ldb=7), dict(ldh=7), dict(lddb=7),
              dict(lddr=7), dict(ldg=7), dict(ldg=8, lddg=7), dict(rows=-1), dict(d=0), dict(rscale=float("nan")), dict(b=None),
              dict(st=None), dict(h=None), dict(dy=None, dh=None), dict(gate=None), dict(flags=0), dict(flags=0, dba=None)):
        assert call(**b) == km.KMP_EINVAL, b
    none = dict(dgate=None, dga=None, dba=None, dg=None, dbe=None)
    assert call(ws=None) == km.KMP_EWORKSPACE and call(n=need - 1) == km.KMP_EWORKSPACE and call(ws=P + 8) == km.KMP_EWORKSPACE
    for k in none:
        assert call(ws=None, **dict(none, **{k: P})) == km.KMP_EWORKSPACE, k
    assert call(db=None, dres=None, ws=None, **none) == km.KMP_OK       # nothing asked for
    size = km.lib().kmp_block_norm_workspace_bytes
    for a in ((0, 1, 1), (4, 1, 1), (1, -1, 1), (1, 1, 0), (1, 1 << 31, 1)):
        assert size(*a) == 0
    assert all(size(t, 0, 1) >= 256 for t in (1, 2, 3))


def test_workspace_does_not_fall(km):  # noqa: F811
    """A workspace of a program's largest call serves its smaller ones."""
    size = km.lib().kmp_block_norm_workspace_bytes
    for t in (1, 2, 3):
        for d in (1, 100, 4096, 8193, 16385, 100000):
            sizes = [size(t, r, d) for r in (0, 1, 5, 63, 64, 500, 511, 4095, 4096, 10000, 100000)]
            assert sizes == sorted(sizes), (t, d, sizes)
        for r in (1, 9, 300, 5000):
            sizes = [size(t, r, d) for d in (1, 255, 256, 257, 512, 513, 2048, 2049, 4096, 4097, 8192, 8193, 16384, 16385, 50000)]
            assert sizes == sorted(sizes), (t, r, sizes)


def test_binding_refuses_tensors(km):  # noqa: F811
    x = torch.zeros(2, 3)
    with pytest.raises(km.KmpError, match="b must be a 2-D device tensor"):
        km.kmp_block_norm(x, x, x, x, 1e-5)
    with pytest.raises(km.KmpError, match="b must be a 2-D device tensor"):
        km.kmp_block_norm_backward(x, x, x, x, None, x, x)


@pytest.mark.parametrize("after", [True, False])
@pytest.mark.parametrize("rms", [True, False])
@pytest.mark.parametrize("gate", ["none", "vector", "matrix"])
def test_oracle_gradients_against_differences(after, rms, gate):
    """Central differences in 64 bits, step 1e-5: errors of the order 1e-10 of the third
    derivatives and 1e-16 / 1e-5 of the values."""
    rng = np.random.default_rng(11)
    rows, d = 3, 7
    p = dict(b=rng.standard_normal((rows, d)), res=rng.standard_normal((rows, d)), gamma=1 + 0.3 * rng.standard_normal(d),
             beta=rng.standard_normal(d))
    if after:
        p.update(gamma_after=1 + 0.3 * rng.standard_normal(d), beta_after=rng.standard_normal(d))
    if gate != "none":
        p["gate"] = rng.standard_normal(d if gate == "vector" else (rows, d))
    cy, ch = rng.standard_normal((rows, d)), rng.standard_normal((rows, d))

    def run(q):
        return OO.block_norm(q["b"], q["res"], q.get("gamma_after"), q.get("beta_after"), q.get("gate"), q["gamma"], q["beta"],
                             1e-5, 0.6, after, rms)

    def loss(q):
        h, y, _ = run(q)
        return (y * cy).sum() + (h * ch).sum()

    h, _, stats = run(p)
    e = OO.block_norm_backward(cy, ch, p["b"], h, stats, p.get("gamma_after"), p.get("beta_after"), p.get("gate"), p["gamma"], 0.6,
                               after, rms)
    for k, v in p.items():
        got = e["d" + k]
        if k == "gate" and gate == "vector":
            got = got.sum(axis=0)
        for i in np.ndindex(v.shape):
            up, down = (dict(p, **{k: v + s * 1e-5 * (np.arange(v.size).reshape(v.shape) == np.ravel_multi_index(i, v.shape))})
                        for s in (1, -1))
            want = (loss(up) - loss(down)) / 2e-5
            assert abs(got[i] - want) <= 1e-6 * (1 + abs(want)), (k, i, got[i], want)


def test_largest_arguments(km):  # noqa: F811
    """Sizes up to the largest accepted ones have a workspace; pointers and pitches there
    are refused or taken without overflow."""
    most = (1 << 31) - 1
    size = km.lib().kmp_block_norm_workspace_bytes
    for t in (1, 2, 3):
        for r, d in ((most, most), (most, 1), (0, most), (1, most)):
            assert size(t, r, d) >= 4 * 4 * d and size(t, r, d) < 1 << 62

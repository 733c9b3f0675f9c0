"""Calls of the norms around a block through the C interface that the binding does not
make, and streams in place: bit for bit what the same call otherwise gives."""
import pytest

from tests.gpu_common import announce, device
from tests.test_gpu_block_norm import EPS, Case

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("d", [6, 640, 1025, 4096, 20001])
def test_no_gate_with_a_leading_dimension(d):
    """Without a gate its leading dimension means nothing: rows in registers, and long ones."""
    import torch
    from paper_2606_06742_amd import kmpath as km
    L, rows, code = km.lib(), 7, km._type(torch.bfloat16, "b")
    flags = km.KMP_NORM_AFTER
    c = Case(rows, d, "bf16", "bf16", True, False, "none")
    p = {k: c.t[k].data_ptr() for k in ("b", "res", "gamma_after", "beta_after", "gamma", "beta")}
    outs = []
    for ldg in (0, d, d + 8):
        announce(f"block norm without a gate, d {d}, leading dimension {ldg}")
        h, y, db, dres = (torch.full((rows, d), float("nan"), dtype=torch.bfloat16, device=device()) for _ in range(4))
        sums = [torch.full((d,), float("nan"), dtype=torch.bfloat16, device=device()) for _ in range(4)]
        stats, ws = torch.empty(rows, 4, device=device()), c.workspace()
        stream = torch.cuda.current_stream().cuda_stream
        assert L.kmp_block_norm(stream, code, flags, p["b"], d, p["res"], d, rows, d, code, p["gamma_after"], p["beta_after"], None,
                                ldg, 0.7, p["gamma"], p["beta"], EPS, h.data_ptr(), d, code, y.data_ptr(), d, stats.data_ptr(),
                                None) == km.KMP_OK
        assert L.kmp_block_norm_backward(stream, code, flags, y.data_ptr(), d, c.t["res"].data_ptr(), d, p["b"], d, h.data_ptr(), d,
                                         rows, d, code, p["gamma_after"], p["beta_after"], None, ldg, 0.7, p["gamma"],
                                         stats.data_ptr(), db.data_ptr(), d, dres.data_ptr(), d, None, 0, *(s.data_ptr() for s in sums),
                                         ws.data_ptr(), ws.numel()) == km.KMP_OK
        outs.append([h, y, db, dres, stats, *sums])
    torch.cuda.synchronize()
    for other in outs[1:]:
        for a, b in zip(outs[0], other):
            assert not a.isnan().any() and torch.equal(a, b)


@pytest.mark.parametrize("xt", ["f32", "bf16"])
@pytest.mark.parametrize("d", [7, 333, 1025, 1031, 4160, 8190, 16391, 17001])
def test_rows_in_8_bits_in_place(xt, d):
    """h over res with y in 8 bits, with and without a norm of b (no barrier then stands
    between a wavefront's first reads of res and another's writes of h): widths that are
    no whole number of vectors, whose last ones overlap their neighbours."""
    import torch
    from tests.test_gpu_operators import _put
    import numpy as np
    rows = 600
    for after, rms in ((False, False), (False, True), (True, False)):
        announce(f"block norm to 8 bits in place {xt} {rows} x {d}, norm of b {after}, root mean square {rms}")
        c = Case(rows, d, xt, xt, after, rms, "vector", rscale=3.0)
        outs = []
        for h in (c.matrix(), c.t["res"]):
            q, _ = _put(np.zeros((rows, d), np.int8), torch.int8)
            scale = torch.full((rows,), float("nan"), device=device())
            c.forward(h, q, scale)
            outs.append((h, q, scale, c.stats.clone()))
        for a, b in zip(*outs):
            assert torch.equal(a, b)


@pytest.mark.parametrize("gate", [None, "vector", "matrix"])
def test_rows_of_2_28_columns(gate):
    """Columns beyond 2^28: more than a launch has threads. Without a norm of b every
    element of h, db and dres has two roundings; a thread adds d / 1024 terms of a sum of a
    row one after another, each within 2^-24 of it: y, db and dres by 2^-6 of the largest."""
    import torch
    from paper_2606_06742_amd import kmpath as km
    rows, d, t = 2, 2 ** 28 + 65, torch.bfloat16
    g = torch.Generator(device=device()).manual_seed(7)
    rand = lambda *n: torch.randn(*n, generator=g, device=device(), dtype=t)
    b, res, dy, dh, gamma = rand(rows, d), rand(rows, d), rand(rows, d), rand(rows, d), rand(d)
    w = None if gate is None else rand(d) if gate == "vector" else rand(rows, d)
    new = lambda *n: torch.full(n, float("nan"), dtype=t, device=device())
    h, y, db, dres, dgamma, dbeta = new(rows, d), new(rows, d), new(rows, d), new(rows, d), new(d), new(d)
    dw = None if w is None else torch.full_like(w, float("nan"))
    stats = torch.full((rows, 4), float("nan"), device=device())
    ws = torch.empty(km.kmp_block_norm_workspace_bytes(rows, d, t), dtype=torch.uint8, device=device())
    form = dict(gate=w, gamma=gamma, rscale=0.5, after=False, rms=True)
    announce(f"block norm {rows} x {d}, gate {gate}")
    km.kmp_block_norm(b, res, h, y, EPS, stats=stats, **form)
    km.kmp_block_norm_backward(dy, dh, b, h, stats, db, dres, dgate=dw, dgamma=dgamma, dbeta=dbeta, workspace=ws, **form)
    one = torch.ones((), device=device())
    near = lambda got, want, off: bool(((got.float() - want).abs() <= off + 2.0 ** -8 * (want.abs() + off)).all())
    sums = [torch.zeros(d, device=device()) for _ in range(3)]
    for r in range(rows):
        wr = one if w is None else (w if w.dim() == 1 else w[r]).float()
        he = 0.5 * res[r].float() + wr * b[r].float()
        assert near(h[r], he, 2.0 ** -22 * 16)
        rs = float(1 / torch.sqrt((he.double() ** 2).mean() + EPS))
        assert abs(float(stats[r, 3]) / rs - 1) < 2.0 ** -6
        assert near(y[r], he * rs * gamma.float(), 2.0 ** -6 * float(he.abs().max()) * rs * float(gamma.abs().max()))
        xh, v = h[r].float() * float(stats[r, 3]), dy[r].float() * gamma.float()
        s = dh[r].float() + float(stats[r, 3]) * (v - xh * float((v.double() * xh.double()).mean()))
        most = 2.0 ** -6 * float(s.abs().max())
        assert near(dres[r], 0.5 * s, most) and near(db[r], wr * s, most * float(wr.abs().max()))
        if gate == "matrix":
            assert near(dw[r], s * b[r].float(), most * float(b.float().abs().max()))
        sums[0] += s * b[r].float()
        sums[1] += dy[r].float() * xh
        sums[2] += dy[r].float()
    assert near(dgamma, sums[1], 2.0 ** -18) and near(dbeta, sums[2], 2.0 ** -20)
    assert gate != "vector" or near(dw, sums[0], 2 * most * float(b.float().abs().max()))


def test_numbers_of_numpy():
    """The scale and eps of any real type, forward as backward."""
    import numpy as np
    import torch
    c = Case(5, 333, "bf16", "f32", True, False, "vector")
    outs = []
    for kind in (float, np.float32, np.float64):
        from paper_2606_06742_amd import kmpath as km
        h, y, db, dres = c.matrix(), c.matrix(), c.matrix(), c.matrix()
        form = dict(c.form(("gamma_after", "beta_after", "gate", "gamma")), rscale=kind(0.75))
        km.kmp_block_norm(c.t["b"], c.t["res"], h, y, kind(2.0 ** -10), beta=c.t["beta"], stats=c.stats, **form)
        km.kmp_block_norm_backward(y, h, c.t["b"], h, c.stats, db, dres, **form)
        outs.append((h, y, db, dres))
    for other in outs[1:]:
        assert all(torch.equal(a, b) for a, b in zip(outs[0], other))

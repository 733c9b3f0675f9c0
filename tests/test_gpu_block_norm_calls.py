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

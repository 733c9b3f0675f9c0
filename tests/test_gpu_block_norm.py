"""The norms around a block on the GPU against oracle/operators.py (64 bits): types,
norms, gates, widths around every form's borders, strides, unaligned rows, missing
operands, non-finite rows, in-place streams, rows in 8 bits, replays from a graph.

Bounds. u = 2^-24 is the unit roundoff of the arithmetic, uo that of the output type.
A sum of d terms over at least 64 lanes is in error by at most (d/64 + 16) u times the
sum of the terms' sizes; a product, quotient or root adds a few u. The bounds below are
first-order sums of such terms."""
import numpy as np
import pytest

from oracle import operators as OO
from tests.gpu_common import announce, device
from tests.test_gpu_operators import TINY, U, _dtype, _hidden, _np, _put

pytestmark = pytest.mark.gpu

EPS = 1e-5
u = U["f32"]
# rows, d, gap between rows, first element's offset
SHAPES = [(1, 1, 0, 0), (3, 2, 1, 1), (5, 7, 0, 0), (2, 64, 0, 0), (9, 255, 0, 1), (3, 257, 3, 0), (2, 511, 0, 0),
          (2, 513, 0, 0), (7, 1024, 8, 0), (2, 1025, 1, 1), (2, 1999, 0, 1), (3, 2048, 0, 0), (2, 2056, 0, 0),
          (1, 4096, 0, 0), (5, 4100, 4, 2), (2, 8192, 0, 0), (2, 8200, 0, 0), (2, 16384, 0, 0), (2, 16385, 0, 1),
          (1, 40009, 0, 0)]
PAIRS = [("f32", "f32"), ("bf16", "bf16"), ("bf16", "f32"), ("f16", "f16"), ("f16", "f32")]


def _out(got, want, bound, t):
    """Every element within its bound and the output type's rounding."""
    uo = U[t] if t != "f32" else u
    return np.all(np.abs(_np(got) - want) <= bound + uo * (np.abs(want) + bound) + TINY[t])


class Case:
    """Inputs of one shape and form, their values in 64 bits, and the calls."""

    def __init__(self, rows, d, xt, wt, after, rms, gate, betas=True, weights=True, rscale=0.7, res=True, pad=0, off=0, seed=0):
        import torch
        self.rng = rng = np.random.default_rng(rows * 100003 + d + seed)
        self.rows, self.d, self.xt, self.wt, self.after, self.rms, self.rscale = rows, d, xt, wt, after, rms, rscale
        self.pad, self.off = pad, off
        self.t, self.v = {}, {}
        self.put("b", _hidden(rng, rows, d))
        if res:
            self.put("res", 2.0 * _hidden(rng, rows, d))
        for k in ("gamma_after", "gamma"):
            if weights:
                self.put(k, 1.0 + 0.2 * rng.standard_normal(d))
        for k in ("beta_after", "beta"):
            if betas:
                self.put(k, 0.1 * rng.standard_normal(d))
        if gate == "vector":
            self.put("gate", 0.5 + 0.3 * rng.standard_normal(d))
        elif gate == "matrix":
            self.put("gate", 0.5 + 0.3 * rng.standard_normal((rows, d)))
        self.stats = torch.empty(rows, 4, device=device())

    def put(self, k, a):
        if a.ndim == 2:
            self.t[k], self.v[k] = _put(a, _dtype(self.xt), self.pad, self.off)
        else:
            t, v = _put(a[None], _dtype(self.wt))
            self.t[k], self.v[k] = t[0], v[0]

    def matrix(self):
        import torch
        pitch = self.d + self.pad
        buf = torch.full((self.rows * pitch + self.off,), float("nan"), dtype=_dtype(self.xt), device=device())
        return buf[self.off:].view(self.rows, pitch)[:, :self.d]

    def form(self, names):
        return dict({k: self.t.get(k) for k in names}, rscale=self.rscale, after=self.after, rms=self.rms)

    def forward(self, h, y, scale=None):
        from paper_2606_06742_amd import kmpath as km
        km.kmp_block_norm(self.t["b"], self.t.get("res"), h, y, EPS, stats=self.stats, scale=scale,
                          **self.form(("gamma_after", "beta_after", "gate", "gamma", "beta")))

    def workspace(self):
        import torch
        from paper_2606_06742_amd import kmpath as km
        return torch.full((km.kmp_block_norm_workspace_bytes(self.rows, self.d, _dtype(self.xt)),), 255, dtype=torch.uint8,
                          device=device())

    def backward(self, dy, dh, h, workspace, names=("db", "dres", "dgate", "dgamma_after", "dbeta_after", "dgamma", "dbeta")):
        """The gradients of what there is, by name."""
        import torch
        from paper_2606_06742_amd import kmpath as km
        out = {}
        for k in names:
            if k in ("db", "dres"):
                out[k] = self.matrix()
            elif k == "dgate":
                if "gate" in self.t:
                    out[k] = self.matrix() if self.t["gate"].dim() == 2 else torch.empty_like(self.t["gate"])
            elif self.after or "after" not in k:
                out[k] = torch.empty(self.d, dtype=_dtype(self.wt), device=device())
        f = self.form(("gamma_after", "beta_after", "gate", "gamma"))
        args = [out.get("db"), out.get("dres")]
        km.kmp_block_norm_backward(dy, dh, self.t["b"], h, self.stats, *args, workspace=workspace,
                                   **{k: v for k, v in out.items() if k not in ("db", "dres")}, **f)
        return out

    def check_forward(self, h, y):
        v, rs = self.v, float(np.float32(self.rscale))
        d = self.d
        he, ye, st = OO.block_norm(v["b"], v.get("res"), v.get("gamma_after"), v.get("beta_after"), v.get("gate"),
                                   v.get("gamma"), v.get("beta"), EPS, rs, self.after, self.rms)
        c = d / 64 + 16
        m1, r1, m2, r2 = (st[:, i:i + 1] for i in range(4))
        ga, ca, g0 = v.get("gamma_after", 1.0), v.get("beta_after", 0.0), v.get("gate", 1.0)
        n = np.abs(v["b"])
        en = np.zeros_like(n)
        if self.after:
            # mu within c u mean|b|, r within (c + 12) u and the square of that
            dmu = 0.0 if self.rms else c * u * np.abs(v["b"]).mean(axis=1, keepdims=True) * r1
            xh = np.abs((v["b"] - m1) * r1)
            n = xh * np.abs(ga) + np.abs(ca)
            en = np.abs(ga) * (dmu + xh * ((c + 12) * u + dmu ** 2)) + 4 * u * n
        eh = np.abs(g0) * en + 3 * u * (np.abs(g0) * n + np.abs(rs * v.get("res", 0.0)))
        bad = []
        if h is not None and not _out(h, he, eh, self.xt):
            bad.append("h")
        # h's error goes into its mean, its variance and y itself
        dmu = 0.0 if self.rms else (c * u * np.abs(he).mean(axis=1, keepdims=True) + eh.mean(axis=1, keepdims=True)) * r2
        xh = np.abs((he - m2) * r2)
        er = (c + 12) * u + r2 * (xh * eh).mean(axis=1, keepdims=True) + dmu ** 2
        g, k = np.abs(v.get("gamma", 1.0)), np.abs(v.get("beta", 0.0))
        ey = g * (r2 * eh + dmu + xh * er) * (1 + 1e-3) + 4 * u * (g * xh + k)
        if y is not None and not _out(y, ye, ey, self.xt):
            bad.append("y")
        got = _np(self.stats)
        if self.after:
            if np.any(np.abs(got[:, 0:1] - m1) > c * u * np.abs(v["b"]).mean(axis=1, keepdims=True) + u * np.abs(m1)) or (
                    np.any(np.abs(got[:, 1:2] / r1 - 1) > (c + 12) * u + (c * u * np.abs(v["b"]).mean(axis=1, keepdims=True) * r1) ** 2)):
                bad.append("stats of b")
        elif not (np.all(got[:, 0] == 0) and np.all(got[:, 1] == 1)):
            bad.append("stats without a norm")
        if y is not None and (np.any(np.abs(got[:, 2:3] - m2) * r2 > dmu + u * np.abs(m2) * r2) or np.any(np.abs(got[:, 3:4] / r2 - 1) > er * (1 + 1e-3))):
            bad.append("stats of h")
        return bad, ey

    def check_backward(self, out, dyv, dhv, hv):
        v, rs, d = self.v, float(np.float32(self.rscale)), self.d
        st = _np(self.stats)
        e = OO.block_norm_backward(dyv, dhv, v["b"], hv, st, v.get("gamma_after"), v.get("beta_after"), v.get("gate"),
                                   v.get("gamma"), rs, self.after, self.rms)
        c = d / 64 + 16
        m1, r1, m2, r2 = (st[:, i:i + 1] for i in range(4))
        mean = lambda a: a.mean(axis=1, keepdims=True)

        def back(w, xh, r):
            """Rounding of a norm's gradient: w within 2u, xh within 2u, the means within (c + 8) u."""
            return u * r * ((c + 16) * (mean(w) + 2 * xh * mean(w * xh)) + 8 * w)

        es = np.zeros_like(v["b"])
        xh2 = dy = np.zeros_like(v["b"])
        if dyv is not None:
            xh2, dy = np.abs((hv - m2) * r2), np.abs(dyv)
            es = back(dy * np.abs(v.get("gamma", 1.0)), xh2, r2) + 2 * u * (np.abs(e["s"]) + (0 if dhv is None else np.abs(dhv)))
        g0, ga, ca = np.abs(v.get("gate", 1.0)), np.abs(v.get("gamma_after", 1.0)), np.abs(v.get("beta_after", 0.0))
        s, t = np.abs(e["s"]), np.abs(e["t"])
        et = g0 * es + 2 * u * t
        xh1 = np.abs((v["b"] - m1) * r1) if self.after else np.abs(v["b"])
        edb = et
        if self.after:
            ew, w = ga * et + u * ga * t, ga * t
            edb = r1 * (ew + mean(ew) + xh1 * mean(xh1 * ew)) * (1 + 1e-3) + back(w, xh1, r1) + 2 * u * np.abs(e["db"])
        per_row = np.ndim(v.get("gate", 0)) == 2
        k = (self.rows + 20) * u
        q, eq = (t, et) if per_row else (s, es)
        ea, eb = (eq * xh1 + k * q * xh1).sum(axis=0), (eq + k * q).sum(axis=0)
        bounds = dict(dres=np.abs(rs) * es + 3 * u * np.abs(e["dres"]), db=edb, dgamma=k * (dy * xh2).sum(axis=0), dbeta=k * dy.sum(axis=0))
        size_a, size_b = (q * xh1).sum(axis=0), q.sum(axis=0)
        f = 1.0 if per_row else g0
        bounds["dgamma_after"], bounds["dbeta_after"] = f * (ea + 3 * u * size_a), f * (eb + 3 * u * size_b)
        want = dict(e)
        if per_row:
            n = xh1 * ga + ca if self.after else xh1
            bounds["dgate"] = es * n + 5 * u * s * n
        else:
            want["dgate"] = e["dgate"].sum(axis=0)
            bounds["dgate"] = (ga * ea + ca * eb + 4 * u * (ga * size_a + ca * size_b)) if self.after else ea
        bad = []
        for name, got in out.items():
            kind = self.xt if got.dim() == 2 else self.wt
            if not _out(got, want[name], bounds[name], kind):
                bad.append(name)
        return bad


FORMS = [(after, rms, gate) for after in (True, False) for rms in (False, True) for gate in ("none", "vector", "matrix")]


@pytest.mark.parametrize("xt,wt", PAIRS)
def test_forward_and_backward(xt, wt):
    """Every shape with some of the forms, every form with some of the shapes."""
    import torch
    for i, (rows, d, pad, off) in enumerate(SHAPES):
        for after, rms, gate in (FORMS if d in (7, 257, 1999) else [FORMS[(5 * i + j) % 12] for j in (0, 3)]):
            announce(f"block norm {xt} weights {wt} {rows} x {d} gap {pad} offset {off} after {after} rms {rms} gate {gate}")
            c = Case(rows, d, xt, wt, after, rms, gate, pad=pad, off=off)
            h, y = c.matrix(), c.matrix()
            c.forward(h, y)
            bad, _ = c.check_forward(h, y)
            assert not bad, bad
            dy, dyv = _put(c.rng.standard_normal((rows, d)) + 0.1, _dtype(xt), pad, off)
            dh, dhv = _put(0.5 * c.rng.standard_normal((rows, d)), _dtype(xt), pad, off)
            out = c.backward(dy, dh, h, c.workspace())
            bad = c.check_backward(out, dyv, dhv, _np(h))
            assert not bad, bad
            # again, and in parts: the same bits
            again = c.backward(dy, dh, h, c.workspace())
            parts = c.backward(dy, dh, h, None, ("db", "dres"))
            parts.update(c.backward(dy, dh, h, c.workspace(), ("dgate", "dbeta_after", "dgamma")))
            assert all(torch.equal(out[k], again[k]) for k in out), [k for k in out if not torch.equal(out[k], again[k])]
            assert all(torch.equal(out[k], parts[k]) for k in parts), [k for k in parts if not torch.equal(out[k], parts[k])]


@pytest.mark.parametrize("rows,d", [(r, d) for r in (1, 33, 700, 2051) for d in (5, 100, 640, 3000, 9000, 20000)
                                    if r * d <= 1 << 23])
def test_sums_over_many_rows(rows, d):
    """Counts of rows around the strips of the sums, in 32 and 16 bits."""
    for xt, after, rms, gate in (("f32", True, False, "vector"), ("bf16", True, True, "matrix"), ("f16", False, False, "none")):
        announce(f"block norm backward {xt} {rows} x {d} after {after} rms {rms} gate {gate}")
        c = Case(rows, d, xt, xt, after, rms, gate)
        h, y = c.matrix(), c.matrix()
        c.forward(h, y)
        bad, _ = c.check_forward(h, y)
        dy, dyv = _put(c.rng.standard_normal((rows, d)) + 0.1, _dtype(xt))
        dh, dhv = _put(0.5 * c.rng.standard_normal((rows, d)), _dtype(xt))
        out = c.backward(dy, dh, h, c.workspace())
        bad += c.check_backward(out, dyv, dhv, _np(h))
        assert not bad, bad


@pytest.mark.parametrize("d", [3, 300, 2500, 33000])
def test_missing_operands(d):
    """Without residual, weights, one of the gradients, one of the outputs."""
    import torch
    rows = 5
    for after, rms, gate in ((True, False, "none"), (False, True, "vector"), (True, True, "matrix")):
        announce(f"block norm, operands missing, {rows} x {d} after {after} rms {rms} gate {gate}")
        c = Case(rows, d, "bf16", "f32", after, rms, gate, betas=False, weights=False, res=False)
        h, y = c.matrix(), c.matrix()
        c.forward(h, y)
        bad, _ = c.check_forward(h, y)
        assert not bad, bad
        stats = c.stats.clone()
        h2, y2 = c.matrix(), c.matrix()
        c.forward(None, y2)
        assert torch.equal(y2, y) and torch.equal(c.stats, stats)
        c.forward(h2, None)
        assert torch.equal(h2, h) and torch.equal(c.stats[:, :2], stats[:, :2])
        assert np.all(_np(c.stats)[:, 2:] == [0.0, 1.0])
        c.stats.copy_(stats)
        g, gv = _put(c.rng.standard_normal((rows, d)), _dtype("bf16"))
        bad = c.check_backward(c.backward(g, None, h, c.workspace()), gv, None, _np(h))
        bad += c.check_backward(c.backward(None, g, None, c.workspace()), None, gv, None)
        assert not bad, bad


@pytest.mark.parametrize("xt", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("d", [5, 333, 4096, 17000])
def test_rows_in_8_bits(xt, d):
    """y in 8 bits: off by a half step of the row's scale and y's own error."""
    import torch
    rows = 6
    c = Case(rows, d, xt, xt, True, d % 2 == 0, "vector")
    h, y = c.matrix(), c.matrix()
    c.forward(h, y)
    _, ey = c.check_forward(h, y)
    announce(f"block norm to 8 bits {xt} {rows} x {d}")
    q, _ = _put(np.zeros((rows, d), np.int8), torch.int8, 3, 1)
    scale = torch.empty(rows, device=device())
    h2 = c.matrix()
    c.forward(h2, q, scale)
    assert torch.equal(h, h2)
    v = c.v
    _, ye, _ = OO.block_norm(v["b"], v["res"], v["gamma_after"], v["beta_after"], v["gate"], v["gamma"], v["beta"], EPS,
                             float(np.float32(c.rscale)), c.after, c.rms)
    sc = _np(scale)
    most = np.abs(ye).max(axis=1)
    assert np.all(np.abs(sc * 127 - most) <= ey.max(axis=1) + 4 * u * most)
    # half a step, the error of y, and the rounding of three products at up to 127
    assert np.all(np.abs(q.double().cpu().numpy() * sc[:, None] - ye) <= sc[:, None] * (0.5 + 127 * 4 * u) + 2 * ey.max(axis=1)[:, None])


def test_stream_in_place_and_no_rows():
    """h written over res; calls of no rows set the sums to zero and touch nothing else."""
    import torch
    from paper_2606_06742_amd import kmpath as km
    for d in (6, 700, 4096, 20001):
        announce(f"block norm in place, d {d}")
        c = Case(7, d, "bf16", "bf16", True, False, "vector")
        h, y, y2 = c.matrix(), c.matrix(), c.matrix()
        c.forward(h, y)
        c.forward(c.t["res"], y2)
        assert torch.equal(c.t["res"], h) and torch.equal(y, y2)
        none = torch.empty(0, d, dtype=torch.bfloat16, device=device())
        sums = [torch.full((d,), 7.0, dtype=torch.bfloat16, device=device()) for _ in range(5)]
        ws = torch.empty(km.kmp_block_norm_workspace_bytes(0, d, torch.bfloat16), dtype=torch.uint8, device=device())
        km.kmp_block_norm(none, none, none, none, EPS)
        km.kmp_block_norm_backward(none, none, none, none, torch.empty(0, 4, device=device()), none, none, gate=c.t["gate"],
                                   dgate=sums[0], dgamma_after=sums[1], dbeta_after=sums[2], dgamma=sums[3], dbeta=sums[4],
                                   workspace=ws)
        assert all(bool((s == 0).all()) for s in sums)


def test_rows_that_are_not_finite():
    """A NaN or an infinity spoils its own row, and the sums over the rows alone."""
    for d in (9, 640, 9000, 20000):
        for bad in (float("nan"), float("inf")):
            announce(f"block norm with {bad}, d {d}")
            c = Case(6, d, "f32", "f32", True, False, "vector", seed=1)
            h, y, h2, y2 = (c.matrix() for _ in range(4))
            c.forward(h, y)
            c.t["b"][2, d // 2] = bad
            c.t["res"][4, d - 1] = bad
            c.forward(h2, y2)
            for r in (0, 1, 3, 5):
                assert bool((h[r] == h2[r]).all()) and bool((y[r] == y2[r]).all())
            assert bool(y2[2].isnan().all()) and bool(y2[4].isnan().any()) and not bool(h2[4, : d - 1].isnan().any())


def test_replayed_from_a_graph():
    """Forward and backward captured and replayed with new inputs and eager calls between."""
    import torch
    c = Case(300, 1500, "bf16", "bf16", True, True, "vector")
    h, y = c.matrix(), c.matrix()
    dy, _ = _put(c.rng.standard_normal((300, 1500)), torch.bfloat16)
    dh, _ = _put(c.rng.standard_normal((300, 1500)), torch.bfloat16)
    ws = c.workspace()
    c.forward(h, y)
    c.backward(dy, dh, h, ws)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        c.forward(h, y)
        out = c.backward(dy, dh, h, ws)
    for i in range(4):
        announce(f"block norm replay {i}")
        c.t["b"].mul_(1.1)
        dy.add_(0.05)
        g.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in (h, y, *out.values())]
        h2, y2 = c.matrix(), c.matrix()
        c.forward(h2, y2)
        eager = c.backward(dy, dh, h2, c.workspace())
        for a, b in zip(got, (h2, y2, *eager.values())):
            assert torch.equal(a, b)


def test_gradients_against_differences():
    """The gradients against differences of the library's own outputs in 32 bits: the loss
    sum of y cy + h ch along random directions, steps of 2^-6 either way. The error of a
    difference is of the order step^2 (about 1e-3 of the gradient here) and the outputs'
    rounding over the step."""
    import torch
    from paper_2606_06742_amd import kmpath as km
    rows, d = 6, 96
    for after, rms, gate in FORMS:
        c = Case(rows, d, "f32", "f32", after, rms, gate, seed=5)
        cy, cyv = _put(c.rng.standard_normal((rows, d)), torch.float32)
        ch, chv = _put(c.rng.standard_normal((rows, d)), torch.float32)
        h, y = c.matrix(), c.matrix()

        def loss():
            c.forward(h, y)
            return float((y.double() * cy.double()).sum() + (h.double() * ch.double()).sum())

        loss()
        out = c.backward(cy, ch, h, c.workspace())
        names = {"db": "b", "dres": "res", "dgate": "gate", "dgamma": "gamma", "dbeta": "beta", "dgamma_after": "gamma_after",
                 "dbeta_after": "beta_after"}
        for k, g in out.items():
            t = c.t[names[k]]
            keep = t.clone()
            step = torch.randn(t.shape, generator=torch.Generator().manual_seed(3)).to(device())
            eps = 2.0 ** -6
            t.copy_(keep + eps * step)
            up = loss()
            t.copy_(keep - eps * step)
            down = loss()
            t.copy_(keep)
            want = float((g.double() * step.double()).sum())
            size = float((g.double() * step.double()).square().sum().sqrt())
            assert abs((up - down) / (2 * eps) - want) <= 2e-2 * size + 1e-2, (after, rms, gate, k, up, down, want, size)

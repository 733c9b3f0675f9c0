"""The operators together as a program uses them: a model's last block and its end,
forward, backward, in 8 bits, and the choice of tokens with their log probabilities.

    a = gelu(layer_norm(x) W1' + b1),  o = a W2' + b2
    h = 0.8 x + gate N(o),  y = N(h),  logits = y W3'

The reference is the same chain in 64 bits with torch's own gradients."""
import numpy as np
import pytest

from oracle import operators as OO
from tests.gpu_common import announce, device
from tests.test_gpu_operators import _np

pytestmark = pytest.mark.gpu

EPS, RSCALE = 1e-5, 0.8
NAMES = ("x", "g0", "c0", "W1", "b1", "W2", "b2", "gate", "ga", "ca", "g", "c", "W3")


def _params(T, d, f, V, dtype, seed=0):
    import torch
    gen = torch.Generator().manual_seed(seed)
    r = lambda *s: torch.randn(*s, generator=gen)
    p = dict(x=r(T, d) + 0.2, g0=1 + 0.2 * r(d), c0=0.1 * r(d), W1=r(f, d) / d ** 0.5, b1=0.2 * r(f), W2=r(d, f) / f ** 0.5,
             b2=0.2 * r(d), gate=0.5 + 0.3 * r(d), ga=1 + 0.2 * r(d), ca=0.1 * r(d), g=1 + 0.2 * r(d), c=0.1 * r(d),
             W3=3.0 * r(V, d) / d ** 0.5)
    return {k: v.to(dtype).to(device()) for k, v in p.items()}


class Block:
    """The chain with its buffers."""

    def __init__(self, p):
        import torch
        from paper_2606_06742_amd import kmpath as km
        self.p = p
        dt = p["x"].dtype
        (T, d), f, V = p["x"].shape, p["W1"].shape[0], p["W3"].shape[0]
        e = lambda *s, dtype=dt: torch.empty(*s, dtype=dtype, device=device())
        f32 = torch.float32
        self.y0, self.mean, self.rstd = e(T, d), e(T, dtype=f32), e(T, dtype=f32)
        self.a, self.z, self.o, self.h, self.y = e(T, f), e(T, f), e(T, d), e(T, d), e(T, d)
        self.stats, self.logits = e(T, 4, dtype=f32), e(T, V)
        self.u, self.tokens, self.drawn = torch.rand(T, device=device()), e(T, dtype=torch.int32), e(T, dtype=f32)
        self.logp, self.entropy, self.lstats = e(T, dtype=f32), e(T, dtype=f32), e(T, 2, dtype=f32)
        self.d = {k: torch.empty_like(v) for k, v in p.items()}
        self.da, self.do, self.dy, self.dy0, self.dx0 = e(T, f), e(T, d), e(T, d), e(T, d), e(T, d)
        sizes = [km.kmp_sample_tokens_workspace_bytes(T, V), km.kmp_token_logprobs_workspace_bytes(T, V),
                 km.kmp_layer_norm_workspace_bytes(T, d, dt), km.kmp_block_norm_workspace_bytes(T, d, dt)]
        sizes += [km.kmp_dense_product_workspace_bytes(T, n, k, dt) for n, k in ((f, d), (d, f), (V, d))]
        self.ws = e(max(sizes), dtype=torch.uint8)

    def forward(self):
        from paper_2606_06742_amd import kmpath as km
        p = self.p
        km.kmp_layer_norm(p["x"], p["g0"], p["c0"], EPS, self.y0, mean=self.mean, rstd=self.rstd)
        km.kmp_dense_product(self.y0, p["W1"], self.a, bias=p["b1"], act="gelu", z=self.z)
        km.kmp_dense_product(self.a, p["W2"], self.o, bias=p["b2"])
        km.kmp_block_norm(self.o, p["x"], self.h, self.y, EPS, gamma_after=p["ga"], beta_after=p["ca"], gate=p["gate"],
                          gamma=p["g"], beta=p["c"], rscale=RSCALE, stats=self.stats)
        km.kmp_dense_product(self.y, p["W3"], self.logits)

    def choose(self, **rules):
        from paper_2606_06742_amd import kmpath as km
        km.kmp_sample_tokens(self.logits, self.u, self.tokens, logp=self.drawn, workspace=self.ws, **rules)
        km.kmp_token_logprobs(self.logits, self.tokens, self.logp, entropy=self.entropy, stats=self.lstats, workspace=self.ws)

    def backward(self, dlogp):
        """Gradients of sum dlogp logp (the tokens given); the logits become theirs."""
        from paper_2606_06742_amd import kmpath as km
        p, d = self.p, self.d
        km.kmp_token_logprobs_backward(self.logits, self.tokens, self.lstats, dlogp, self.logits)
        km.kmp_dense_product_backward(self.logits, self.y, p["W3"], None, self.dy, d["W3"], None, workspace=self.ws)
        km.kmp_block_norm_backward(self.dy, None, self.o, self.h, self.stats, self.do, self.dx0, gamma_after=p["ga"],
                                   beta_after=p["ca"], gate=p["gate"], gamma=p["g"], rscale=RSCALE, dgate=d["gate"],
                                   dgamma_after=d["ga"], dbeta_after=d["ca"], dgamma=d["g"], dbeta=d["c"], workspace=self.ws)
        km.kmp_dense_product_backward(self.do, self.a, p["W2"], None, self.da, d["W2"], d["b2"], workspace=self.ws)
        km.kmp_dense_product_backward(self.da, self.y0, p["W1"], self.z, self.dy0, d["W1"], d["b1"], act="gelu", workspace=self.ws)
        km.kmp_layer_norm_backward(self.dy0, p["x"], p["g0"], self.mean, self.rstd, d["x"], d["g0"], d["c0"], self.ws)
        d["x"].add_(self.dx0)


def _reference(p):
    import torch
    q = {k: v.double().cpu().requires_grad_() for k, v in p.items()}
    norm = lambda t, g, c: (t - t.mean(1, keepdim=True)) / torch.sqrt(t.var(1, unbiased=False, keepdim=True) + EPS) * g + c
    a = torch.nn.functional.gelu(norm(q["x"], q["g0"], q["c0"]) @ q["W1"].t() + q["b1"])
    o = a @ q["W2"].t() + q["b2"]
    h = RSCALE * q["x"] + q["gate"] * norm(o, q["ga"], q["ca"])
    return q, norm(h, q["g"], q["c"]) @ q["W3"].t()


@pytest.mark.parametrize("T", [1, 7, 45, 130])
def test_a_training_step_in_32_bits(T):
    """Every gradient against 64 bits: nine operators in a row, each with sums of up to 3001
    terms in error by at most about sqrt(3001) 2^-24 = 3.3e-6 of their size in the mean, and
    norms that carry errors on by less than twice: below 2e-4 with room."""
    import torch
    p = _params(T, 250, 523, 3001, torch.float32, seed=T)
    b = Block(p)
    announce(f"training step of a block, {T} tokens")
    b.forward()
    b.choose(temperature=torch.full((T,), 0.9, device=device()), top_p=torch.full((T,), 0.95, device=device()))
    q, logits = _reference(p)
    # the drawn token is the one that the rules give for these logits, and has its probability
    te, le, margin = OO.sample_tokens(_np(b.logits), _np(b.u), [float(np.float32(0.9))] * T, None, [float(np.float32(0.95))] * T)
    assert np.all(margin > 3001 * 2.0 ** -46) and np.array_equal(b.tokens.cpu().numpy(), te)
    assert np.all(np.abs(_np(b.drawn) - le) <= 2.0 ** -23 * np.abs(le) + 1e-9)
    assert float((b.logits.double().cpu() - logits.detach()).norm() / logits.detach().norm()) <= 2e-4
    tokens = b.tokens.long().cpu()
    lp = torch.log_softmax(logits, 1)[torch.arange(T), tokens]
    assert np.all(np.abs(_np(b.logp) - lp.detach().numpy()) <= 2e-4 * (1 + np.abs(lp.detach().numpy())))
    w = torch.linspace(-1.0, 1.0, T) + 0.3
    grads = torch.autograd.grad((lp * w.double()).sum(), [q[k] for k in NAMES])
    b.backward(w.to(device()))
    for k, g in zip(NAMES, grads):
        err = float((b.d[k].double().cpu() - g).norm() / g.norm())
        assert err <= 2e-4, (k, err)


def test_an_answer_in_16_bits_with_an_8_bit_head():
    """The block norm's rows in 8 bits go into the 8-bit head, tokens are drawn from its
    logits: the same draws as the oracle makes from these logits; the logits within the 8-bit
    rounding (half a step of 1/127 of a row's and a channel's largest, of random sign) of
    the ones in 64 bits."""
    import torch
    from paper_2606_06742_amd import kmpath as km
    for dtype in (torch.bfloat16, torch.float16):
        T, d, V = 33, 512, 8003
        announce(f"an answer with an 8-bit head, {dtype}")
        p = _params(T, d, 1100, V, dtype, seed=3)
        b = Block(p)
        b.forward()
        wq, ws = torch.empty(V, d, dtype=torch.int8, device=device()), torch.empty(V, device=device())
        km.kmp_quantize_rows(p["W3"], wq, ws)
        yq, ys = torch.empty(T, d, dtype=torch.int8, device=device()), torch.empty(T, device=device())
        h2, out = torch.empty_like(b.h), torch.empty(T, V, device=device())
        km.kmp_block_norm(b.o, p["x"], h2, yq, EPS, gamma_after=p["ga"], beta_after=p["ca"], gate=p["gate"], gamma=p["g"],
                          beta=p["c"], rscale=RSCALE, scale=ys)
        assert torch.equal(h2, b.h)
        km.kmp_quantized_product(yq, ys, wq, ws, out)
        y = _np(b.y)
        want = y @ _np(p["W3"]).T
        # errors of both operands, independent, uniform within half a step, and y's own rounding
        step = np.sqrt((_np(ys)[:, None] ** 2 / 12) * (_np(p["W3"]) ** 2).sum(1)[None, :] +
                       (_np(ws)[None, :] ** 2 / 12) * (y ** 2).sum(1)[:, None])
        assert np.all(np.abs(_np(out) - want) <= 8 * step + 2.0 ** -6 * np.sqrt((y ** 2).sum(1))[:, None])
        top = torch.full((T,), 40, dtype=torch.int32, device=device())
        km.kmp_sample_tokens(out, b.u, b.tokens, top_k=top, logp=b.drawn, workspace=b.ws)
        te, _, margin = OO.sample_tokens(_np(out), _np(b.u), None, [40] * T)
        assert np.all(margin > V * 2.0 ** -46) and np.array_equal(b.tokens.cpu().numpy(), te)


def test_the_run_from_a_graph():
    """Forward, choice and backward in one graph, replayed with new inputs and eager runs
    between, while an eager graph of the same leaves lives."""
    import torch
    p = _params(20, 384, 640, 5000, torch.bfloat16, seed=9)
    b, eager = Block(p), Block(p)
    dlogp = torch.linspace(-1, 1, 20, device=device())
    top_p = torch.full((20,), 0.9, device=device())

    def run(c):
        c.forward()
        c.choose(top_p=top_p)
        c.backward(dlogp)

    run(b)
    torch.cuda.synchronize()
    g, g2 = torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        run(b)
    with torch.cuda.graph(g2):                    # the same buffers and workspace in a second graph
        run(b)
    for i in range(4):
        announce(f"replay {i} of a block's run")
        p["x"].mul_(1.05)
        b.u.copy_(torch.rand(20, device=device()))
        eager.u.copy_(b.u)
        (g if i % 2 == 0 else g2).replay()
        torch.cuda.synchronize()
        run(eager)
        assert torch.equal(b.tokens, eager.tokens) and torch.equal(b.logp, eager.logp)
        for k in NAMES:
            assert torch.equal(b.d[k], eager.d[k]), k


def test_on_another_stream():
    """The run on a stream of its own, handed over explicitly, between the current one's."""
    import torch
    from paper_2606_06742_amd import kmpath as km
    p = _params(9, 200, 300, 2000, torch.float32, seed=4)
    b = Block(p)
    b.forward()
    want = [t.clone() for t in (b.z, b.h, b.y, b.logits)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    for t in (b.z, b.h, b.y, b.logits, b.tokens):
        t.zero_()
    side.wait_stream(torch.cuda.current_stream())
    announce("a block's run on another stream")
    km.kmp_layer_norm(p["x"], p["g0"], p["c0"], EPS, b.y0, mean=b.mean, rstd=b.rstd, stream=side)
    km.kmp_dense_product(b.y0, p["W1"], b.a, bias=p["b1"], act="gelu", z=b.z, stream=side)
    km.kmp_dense_product(b.a, p["W2"], b.o, bias=p["b2"], stream=side)
    km.kmp_block_norm(b.o, p["x"], b.h, b.y, EPS, gamma_after=p["ga"], beta_after=p["ca"], gate=p["gate"], gamma=p["g"],
                      beta=p["c"], rscale=RSCALE, stats=b.stats, stream=side)
    km.kmp_dense_product(b.y, p["W3"], b.logits, stream=side)
    km.kmp_sample_tokens(b.logits, b.u, b.tokens, workspace=b.ws, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(s, t) for s, t in zip(want, (b.z, b.h, b.y, b.logits)))
    assert bool((b.tokens >= 0).all())

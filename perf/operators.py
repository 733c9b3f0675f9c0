"""Performance cases of the operators at a language model's end: the layer norm
(forward, and forward with backward), the 8-bit matrix product with scales for
tokens and channels, and the log probabilities of given tokens with entropy, top
alternatives and gradient.

A case is a dict of plain values with a "kind":

  norm      layer norm of rows, as it is served
  norm_step layer norm forward and backward, as it is trained: y, dx, dgamma, dbeta
  linear    rows quantised to 8 bits and multiplied with 8-bit weights
  head      layer norm with 8-bit rows, and their product with 8-bit weights
  logprobs  log probabilities of tokens, entropy, top alternatives
  loss_step log probabilities and entropy, and the gradient of the logits

listed() holds twelve of them, draw(rng) makes more over the same ranges.
prepare(case, seed) makes what the program has in hand, run(state) is one pass:
in plain torch in 32 bits, or with own = True by the library. exact(case, seed)
gives the same results in 64 bits.
"""
from __future__ import annotations

import math

import torch

own = False

EPS = 1e-5
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
SIZE = {"f32": 4, "bf16": 2, "f16": 2}
# the largest listed cases' elements and products: drawn cases stay below them
MAX_ELEMENTS, MAX_PRODUCTS, MAX_LOGITS, MAX_STEP_LOGITS = 1 << 26, 1 << 38, 2048 * 128000, 1 << 27


def listed():
    return [
        # the norm of one new token
        dict(name="norm_token", kind="norm", type="bf16", weights="same", rows=1, d=4096),
        # the features of a data set of ten thousand points, narrow rows
        dict(name="norm_features", kind="norm", type="f32", weights="same", rows=10000, d=100),
        # a training step of a probe with odd sizes
        dict(name="norm_step_odd", kind="norm_step", type="f32", weights="same", rows=1003, d=1999),
        # the training batch of a wide model
        dict(name="norm_step_large", kind="norm_step", type="bf16", weights="f32", rows=16384, d=4096),
        # one new token through a projection: the weights are read once
        dict(name="linear_token", kind="linear", type="bf16", out="bf16", M=1, K=4096, N=4096, bias=False),
        # a ragged batch of tokens being decoded
        dict(name="linear_batch", kind="linear", type="f16", out="f32", M=37, K=2051, N=8191, bias=True),
        # a long prompt through a wide projection
        dict(name="linear_prompt", kind="linear", type="bf16", out="bf16", M=4096, K=4096, N=16384, bias=False),
        # the end of a decoding step: last norm and vocabulary head for a batch
        dict(name="head_batch", kind="head", type="bf16", weights="same", out="bf16", M=64, K=2048, N=32000),
        # the choice of a few tokens being decoded, with twenty alternatives each
        dict(name="logprobs_tokens", kind="logprobs", type="f32", T=3, V=32000, top=20),
        # scoring the tokens of a long document
        dict(name="logprobs_prompt", kind="logprobs", type="bf16", T=2048, V=128000, top=5),
        # a fine-tuning step on a few hundred tokens, odd vocabulary
        dict(name="loss_step_odd", kind="loss_step", type="f32", T=333, V=40009),
        # the loss of a training batch
        dict(name="loss_step_large", kind="loss_step", type="bf16", T=2048, V=65536),
    ]


def _log_int(rng, lo, hi):
    n = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    return n + 1 if n == 3072 else n


def draw(rng):
    kind = rng.choice(["norm", "norm_step", "linear", "linear", "head", "logprobs", "loss_step"])
    dtype = rng.choice(["bf16", "bf16", "f16", "f32"])
    if kind in ("norm", "norm_step"):
        d = _log_int(rng, 64, 16384)
        # elements of four bytes count twice
        rows = _log_int(rng, 1, max(2, min(16384, MAX_ELEMENTS * 2 // SIZE[dtype] // d)))
        return dict(kind=kind, type=dtype, weights=rng.choice(["same", "f32"]), rows=rows, d=d)
    if kind in ("linear", "head"):
        K, N = _log_int(rng, 64, 12288), _log_int(rng, 64, 32768)
        M = _log_int(rng, 1, max(2, min(8192, MAX_PRODUCTS // (K * N))))
        c = dict(kind=kind, type=dtype, out=dtype if kind == "head" else rng.choice([dtype, "f32"]), M=M, K=K, N=N)
        if kind == "head":
            c["weights"] = "same"
            c["out"] = "bf16" if dtype == "f32" else dtype
        else:
            c["bias"] = rng.random() < 0.3
        return c
    V = _log_int(rng, 1000, 160000)
    most = MAX_LOGITS if kind == "logprobs" else MAX_STEP_LOGITS
    T = _log_int(rng, 1, max(2, min(8192, most * 2 // SIZE[dtype] // V)))
    c = dict(kind=kind, type=dtype, T=T, V=V)
    if kind == "logprobs":
        c["top"] = rng.choice([0, 1, 5, 20])
    return c


# ------------------------------------------------------------------ inputs
def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))
    return g


def _randn(g, *shape):
    return torch.randn(*shape, generator=g, device="cuda")


def _hidden(g, rows, d, dtype):
    """Hidden states: an offset, channels of uneven size, a few large ones."""
    channel = torch.exp(0.5 * _randn(g, d))
    channel[torch.randint(0, d, (max(1, d // 500),), generator=g, device="cuda")] *= 8.0
    return (_randn(g, rows, d) * channel + 0.3 * _randn(g, d)).to(dtype)


def _norm_weights(g, d, dtype):
    return (1.0 + 0.2 * _randn(g, d)).to(dtype), (0.1 * _randn(g, d)).to(dtype)


def _byte_weights(g, N, K):
    """Weights rounded to 8 bits with a scale per channel, each channel's row
    starting at a multiple of 64 bytes (K of the row's bytes are the weights)."""
    W = _randn(g, N, K) * (0.7 + 0.6 * torch.rand(N, 1, generator=g, device="cuda")) / math.sqrt(K)
    scale = W.abs().amax(dim=1) / 127.0
    wq = torch.zeros(N, (K + 63) // 64 * 64, dtype=torch.int8, device="cuda")
    wq[:, :K] = torch.round(W / scale[:, None]).to(torch.int8)
    return wq[:, :K], scale


def _logits(g, T, V, dtype):
    """Logits with a few likely tokens per row, and every 97th row's last
    eighth of the vocabulary ruled out; the targets mostly likely tokens."""
    x = 2.0 * _randn(g, T, V)
    likely = torch.randint(0, V, (T, 8), generator=g, device="cuda")
    x.scatter_add_(1, likely, 6.0 + 3.0 * _randn(g, T, 8))
    x[::97, V - V // 8:] = float("-inf")
    tokens = likely[:, 0].clone()
    tokens[1::3] = torch.randint(0, V - V // 8, (len(tokens[1::3]),), generator=g, device="cuda")
    tokens[2::50] = -1                           # no target (padding, prompts)
    return x.to(dtype), tokens


def prepare(case, seed):
    c, g = case, _gen(seed)
    s = {"case": c}
    dtype = TYPES[c["type"]]
    if c["kind"] in ("norm", "norm_step"):
        s["x"] = _hidden(g, c["rows"], c["d"], dtype)
        s["gamma"], s["beta"] = _norm_weights(g, c["d"], dtype if c["weights"] == "same" else torch.float32)
        if c["kind"] == "norm_step":
            s["dy"] = (_randn(g, c["rows"], c["d"]) + 0.1 * _randn(g, c["d"])).to(dtype)
    elif c["kind"] in ("linear", "head"):
        s["x"] = _hidden(g, c["M"], c["K"], dtype)
        s["wq"], s["wscale"] = _byte_weights(g, c["N"], c["K"])
        if c["kind"] == "head":
            s["gamma"], s["beta"] = _norm_weights(g, c["K"], dtype)
        s["bias"] = 0.1 * _randn(g, c["N"]) if c.get("bias") else None
    else:
        s["logits"], s["tokens"] = _logits(g, c["T"], c["V"], dtype)
        if c["kind"] == "loss_step":
            s["dlogp"] = (-1.0 + 0.3 * _randn(g, c["T"])) / c["T"]
            s["dentropy"] = 0.01 * _randn(g, c["T"]) / c["T"]
    return s


# ------------------------------------------------------- plain forms, 32 bits
def _plain_norm(x, gamma, beta):
    x = x.float()
    mean = x.mean(dim=1, keepdim=True)
    rstd = torch.rsqrt((x - mean).square().mean(dim=1, keepdim=True) + EPS)
    xh = (x - mean) * rstd
    return xh * gamma.float() + beta.float(), xh, rstd


def _plain_product(x, wq, wscale, bias):
    most = x.abs().amax(dim=1, keepdim=True)
    q = torch.round(x * torch.where(most > 0, 127.0 / most, 0.0))
    y = (q @ wq.float().t()) * (most / 127.0) * wscale
    return y if bias is None else y + bias


def _plain_top(x, k):
    """The k largest of each row, equal ones by the lowest index first: the
    order of the values' bits above the complemented index."""
    bits = (x + 0.0).view(torch.int32).long() & 0xFFFFFFFF
    order = torch.where(bits >= 0x80000000, 0xFFFFFFFF - bits, bits + 0x80000000)
    index = torch.arange(x.shape[1], device=x.device)
    key = ((order - 0x80000000) << 32) + (0xFFFFFFFF - index)
    return 0xFFFFFFFF - (torch.topk(key, k, dim=1).values & 0xFFFFFFFF)


def _plain_logprobs(x, tokens):
    m = x.amax(dim=1, keepdim=True)
    m = torch.where(m == float("-inf"), 0.0, m)
    e = torch.exp(x - m)
    s = e.sum(dim=1)
    spread = torch.where(e > 0, e * (x - m), 0.0).sum(dim=1) / s
    lse = m[:, 0] + torch.log(s)
    entropy = torch.where(s > 0, torch.log(s) - spread, 0.0)
    at = x.gather(1, tokens.clamp(min=0)[:, None])[:, 0]
    return torch.where(tokens >= 0, at - lse, 0.0), entropy, lse


def _plain_run(s):
    c = s["case"]
    dtype = TYPES[c["type"]]
    if c["kind"] == "norm":
        return _plain_norm(s["x"], s["gamma"], s["beta"])[0].to(dtype)
    if c["kind"] == "norm_step":
        y, xh, rstd = _plain_norm(s["x"], s["gamma"], s["beta"])
        dy = s["dy"].float()
        w = dy * s["gamma"].float()
        dx = (w - w.mean(dim=1, keepdim=True) - xh * (w * xh).mean(dim=1, keepdim=True)) * rstd
        wt = s["gamma"].dtype
        return y.to(dtype), dx.to(dtype), (dy * xh).sum(dim=0).to(wt), dy.sum(dim=0).to(wt)
    if c["kind"] == "linear":
        return _plain_product(s["x"].float(), s["wq"], s["wscale"], s["bias"]).to(TYPES[c["out"]])
    if c["kind"] == "head":
        y = _plain_norm(s["x"], s["gamma"], s["beta"])[0]
        return _plain_product(y, s["wq"], s["wscale"], None).to(TYPES[c["out"]])
    x, tokens = s["logits"].float(), s["tokens"]
    logp, entropy, lse = _plain_logprobs(x, tokens)
    if c["kind"] == "logprobs":
        ids = _plain_top(x, c["top"]) if c["top"] else tokens.new_empty(c["T"], 0)
        return logp, entropy, ids.int(), x.gather(1, ids) - lse[:, None]
    g = torch.where(tokens >= 0, s["dlogp"], 0.0)[:, None]
    h = s["dentropy"][:, None]
    lp = x - lse[:, None]
    p = torch.exp(lp)
    dx = torch.where(p > 0, -p * (g + h * (lp + entropy[:, None])), 0.0)
    dx.scatter_add_(1, tokens.clamp(min=0)[:, None], g)
    return logp, entropy, dx.to(dtype)


# ---------------------------------------------------------- the library's calls
def _empty(*shape, dtype=torch.float32):
    return torch.empty(*shape, dtype=dtype, device="cuda")


def _buffers(s, km):
    """The outputs and workspaces that a program keeps from call to call."""
    c = s["case"]
    dtype = TYPES[c["type"]]
    b = {}
    if c["kind"] in ("norm", "norm_step"):
        rows, d = c["rows"], c["d"]
        b["y"] = _empty(rows, d, dtype=dtype)
        if c["kind"] == "norm_step":
            b["mean"], b["rstd"] = _empty(rows), _empty(rows)
            b["dx"] = _empty(rows, d, dtype=dtype)
            b["dgamma"], b["dbeta"] = torch.empty_like(s["gamma"]), torch.empty_like(s["beta"])
            b["ws"] = _empty(km.kmp_layer_norm_workspace_bytes(rows, d, dtype), dtype=torch.uint8)
    elif c["kind"] in ("linear", "head"):
        b["q"] = _empty(c["M"], (c["K"] + 63) // 64 * 64, dtype=torch.int8)[:, :c["K"]]
        b["scale"] = _empty(c["M"])
        b["y"] = _empty(c["M"], c["N"], dtype=TYPES[c["out"]])
    else:
        T, top = c["T"], c.get("top", 0)
        b["logp"], b["entropy"] = _empty(T), _empty(T)
        b["top_id"], b["top_logp"] = _empty(T, top, dtype=torch.int32), _empty(T, top)
        b["ws"] = _empty(km.kmp_token_logprobs_workspace_bytes(T, c["V"], top), dtype=torch.uint8)
        if c["kind"] == "loss_step":
            b["stats"], b["dx"] = _empty(T, 2), _empty(T, c["V"], dtype=dtype)
    return b


def _own_run(s):
    from paper_2606_06742_amd import kmpath as km
    kind = s["case"]["kind"]
    if "buffers" not in s:
        s["buffers"] = _buffers(s, km)
    b = s["buffers"]
    if kind == "norm":
        km.kmp_layer_norm(s["x"], s["gamma"], s["beta"], EPS, b["y"])
        return b["y"]
    if kind == "norm_step":
        km.kmp_layer_norm(s["x"], s["gamma"], s["beta"], EPS, b["y"], mean=b["mean"], rstd=b["rstd"])
        km.kmp_layer_norm_backward(s["dy"], s["x"], s["gamma"], b["mean"], b["rstd"], b["dx"], b["dgamma"],
                                   b["dbeta"], b["ws"])
        return b["y"], b["dx"], b["dgamma"], b["dbeta"]
    if kind in ("linear", "head"):
        if kind == "linear":
            km.kmp_quantize_rows(s["x"], b["q"], b["scale"])
        else:
            km.kmp_layer_norm(s["x"], s["gamma"], s["beta"], EPS, b["q"], scale=b["scale"])
        km.kmp_quantized_product(b["q"], b["scale"], s["wq"], s["wscale"], b["y"], bias=s["bias"])
        return b["y"]
    if kind == "logprobs":
        km.kmp_token_logprobs(s["logits"], s["tokens"], b["logp"], entropy=b["entropy"], top_id=b["top_id"],
                              top_logp=b["top_logp"], workspace=b["ws"])
        return b["logp"], b["entropy"], b["top_id"], b["top_logp"]
    km.kmp_token_logprobs(s["logits"], s["tokens"], b["logp"], entropy=b["entropy"], stats=b["stats"],
                          workspace=b["ws"])
    km.kmp_token_logprobs_backward(s["logits"], s["tokens"], b["stats"], s["dlogp"], b["dx"],
                                   entropy=b["entropy"], dentropy=s["dentropy"])
    return b["logp"], b["entropy"], b["dx"]


def run(state):
    return _own_run(state) if own else _plain_run(state)


def work(case):
    c = case
    b = SIZE[c["type"]]
    if c["kind"] in ("norm", "norm_step"):
        n = c["rows"] * c["d"]
        wb = b if c["weights"] == "same" else 4
        if c["kind"] == "norm":
            return {"bytes": 2 * b * n + 2 * wb * c["d"], "flops": 8 * n}
        return {"bytes": 4 * b * n + 4 * wb * c["d"], "flops": 22 * n}
    if c["kind"] in ("linear", "head"):
        M, K, N = c["M"], c["K"], c["N"]
        extra = 2 * b * K if c["kind"] == "head" else 4 * N if c["bias"] else 0
        return {"bytes": b * M * K + K * N + 4 * N + SIZE[c["out"]] * M * N + extra, "flops": 2 * M * K * N}
    n = c["T"] * c["V"]
    if c["kind"] == "logprobs":
        return {"bytes": b * n + c["T"] * (16 + 8 * c["top"]), "flops": 6 * n}
    return {"bytes": 2 * b * n + 24 * c["T"], "flops": 14 * n}


# -------------------------------------------------------------- 64-bit results
def _exact_norm(x, gamma, beta):
    second, first = (x * x).mean(dim=1, keepdim=True), x.mean(dim=1, keepdim=True)
    return (x - first) / torch.sqrt(second - first * first + EPS) * gamma + beta


def _exact_product(x, s):
    top = x.abs().max(dim=1, keepdim=True).values
    q = torch.where(top > 0, x * 127.0 / top, 0.0).round()
    y = torch.matmul(q, s["wq"].double().t().contiguous()) * s["wscale"].double() * (top / 127.0)
    return y if s["bias"] is None else y + s["bias"].double()


def exact(case, seed):
    s = prepare(case, seed)
    c = case
    if c["kind"] in ("norm", "norm_step"):
        x, gamma, beta = (s[k].double().requires_grad_() for k in ("x", "gamma", "beta"))
        y = _exact_norm(x, gamma, beta)
        if c["kind"] == "norm":
            return y.detach()
        return (y.detach(),) + torch.autograd.grad(y, (x, gamma, beta), s["dy"].double())
    if c["kind"] == "linear":
        return _exact_product(s["x"].double(), s)
    if c["kind"] == "head":
        return _exact_product(_exact_norm(s["x"].double(), s["gamma"].double(), s["beta"].double()), s)
    x, tokens = s["logits"].double(), s["tokens"]
    has = tokens >= 0
    logp, entropy, tops, grads = [], [], [], []
    for r in range(0, c["T"], 512):              # in parts, for memory
        xr = x[r:r + 512].clone().requires_grad_(c["kind"] == "loss_step")
        lse = torch.logsumexp(xr, dim=1)
        lp = xr - lse[:, None]
        H = -(lp.exp() * lp.masked_fill(lp == float("-inf"), 0.0)).sum(dim=1)
        tr, hr = tokens[r:r + 512], has[r:r + 512]
        at = torch.where(hr, lp[torch.arange(len(tr), device=tr.device), tr.clamp(min=0)], 0.0)
        if c["kind"] == "loss_step":
            total = (at * s["dlogp"][r:r + 512].double()).sum() + (H * s["dentropy"][r:r + 512].double()).sum()
            grads.append(torch.autograd.grad(total, xr)[0])
        else:
            tops.append(torch.sort(lp, dim=1, descending=True).values[:, :c["top"]])
        logp.append(at.detach())
        entropy.append(H.detach())
    logp, entropy = torch.cat(logp), torch.cat(entropy)
    if c["kind"] == "loss_step":
        return logp, entropy, torch.cat(grads)
    return logp, entropy, None, torch.cat(tops)

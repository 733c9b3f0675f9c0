"""Performance cases of the operators around a model's last block and of the choice
of its tokens: the norms before and after a block fused with its gate and the
residual's scale, the matrix product with bias, activation and residual in its
epilogue, and sampling of tokens from given random numbers.

A case is a dict of plain values with a "kind":

  block        h = rscale res + gate N(b) and y = N(h), as it is served
  block_step   the same forward and backward, as it is trained
  product      out = act(x W' + bias) + residual
  product_grad gradients of x, W and bias from dout and the saved z = x W' + bias
  sample       tokens drawn with temperature, top-k, top-p and min-p per row, and
               their log probabilities under what was left to draw from

listed() holds twelve of them, draw(rng) makes more over the same ranges.
prepare(case, seed) makes what the program has in hand, run(state) is one pass:
in plain torch in 32 bits (sampling in 64), or with own = True by the library.
exact(case, seed) gives the same results in 64 bits.
"""
from __future__ import annotations

import math

import torch

own = False

EPS = 1e-5
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
SIZE = {"f32": 4, "bf16": 2, "f16": 2}
# the largest listed cases' elements (of two bytes), products and logits: drawn
# cases stay below them
MAX_ELEMENTS, MAX_PRODUCTS, MAX_LOGITS = 1 << 26, 1 << 37, 1024 * 128000


def _block(kind, type, norm, after, gate, rscale, beta, rows, d):
    return dict(kind=kind, type=type, norm=norm, after=after, gate=gate, rscale=rscale, beta=beta, rows=rows, d=d)


def _product(kind, type, act, bias, residual, M, K, N):
    return dict(kind=kind, type=type, act=act, bias=bias, residual=residual, M=M, K=K, N=N)


def _sample(type, T, V, temperature, top_k, top_p, min_p):
    return dict(kind="sample", type=type, T=T, V=V, temperature=temperature, top_k=top_k, top_p=top_p, min_p=min_p)


def listed():
    return [
        # one new token between two blocks
        dict(_block("block", "bf16", "rms", True, "vector", 1.0, False, 1, 4096), name="block_token"),
        # a long prompt between two blocks, a gate per token
        dict(_block("block", "f16", "layer", True, "matrix", 0.5, True, 4096, 5120), name="block_prompt"),
        # a training step of a small model with an odd width
        dict(_block("block_step", "f32", "layer", True, "vector", 1.0, True, 1003, 1999), name="block_step_odd"),
        # the training batch of a wide model
        dict(_block("block_step", "bf16", "rms", True, "vector", 0.7, False, 16384, 4096), name="block_step_large"),
        # one new token through a block's first product: the weights are read once
        dict(_product("product", "bf16", "silu", False, False, 1, 4096, 16384), name="product_token"),
        # a ragged batch of tokens through a block's last product
        dict(_product("product", "f16", "none", True, True, 77, 8191, 2051), name="product_batch"),
        # a long prompt through a block's first product
        dict(_product("product", "bf16", "gelu_tanh", True, False, 4096, 4096, 8192), name="product_prompt"),
        # the gradients of a few hundred tokens in 32 bits, odd sizes
        dict(_product("product_grad", "f32", "gelu", True, False, 509, 1001, 2003), name="product_grad_odd"),
        # the gradients of a training batch
        dict(_product("product_grad", "bf16", "gelu_tanh", True, False, 4096, 4096, 4096), name="product_grad_large"),
        # the next token of one answer
        dict(_sample("f32", 1, 32000, 0.8, 0, 0.95, 0.0), name="sample_token"),
        # the next tokens of a batch of answers, from few tokens each
        dict(_sample("bf16", 64, 128000, 0.7, 50, 0.9, 0.0), name="sample_batch"),
        # many answers of many questions, from many tokens each
        dict(_sample("bf16", 1024, 128000, 1.0, 0, 0.98, 0.001), name="sample_many"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["block", "block_step", "product", "product", "product_grad", "sample", "sample"])
    dtype = rng.choice(["bf16", "bf16", "f16", "f32"])
    if kind in ("block", "block_step"):
        d = _log_int(rng, 64, 16384)
        most = MAX_ELEMENTS * 2 // SIZE[dtype] // (1 if kind == "block_step" else 4)
        return _block(kind, dtype, rng.choice(["rms", "layer"]), rng.random() < 0.7,
                      rng.choice(["none", "vector", "matrix"]), rng.choice([1.0, 0.5, 0.7]), rng.random() < 0.5,
                      _log_int(rng, 1, max(2, min(16384, most // d))), d)
    if kind in ("product", "product_grad"):
        K, N = _log_int(rng, 64, 12288), _log_int(rng, 64, 16384)
        # 32-bit products have a fraction of the rate
        most = MAX_PRODUCTS // (2 if kind == "product_grad" else 1) // (16 if dtype == "f32" else 1)
        M = _log_int(rng, 1, max(2, min(8192, most // (K * N))))
        return _product(kind, dtype, rng.choice(["none", "relu", "gelu", "gelu_tanh", "silu"]), rng.random() < 0.5,
                        kind == "product" and rng.random() < 0.4, M, K, N)
    V = _log_int(rng, 1000, 160000)
    T = _log_int(rng, 1, max(2, min(2048, MAX_LOGITS * 2 // SIZE[dtype] // V)))
    return _sample(dtype, T, V, round(rng.uniform(0.5, 1.5), 2), rng.choice([0, 0, 1, 20, 50, 200, 1000]),
                   rng.choice([1.0, 0.98, 0.95, 0.9, 0.5]), rng.choice([0.0, 0.0, 0.001, 0.05]))


# ------------------------------------------------------------------ inputs
def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))
    return g


def _randn(g, *shape):
    return torch.randn(*shape, generator=g, device="cuda")


def _rand(g, *shape):
    return torch.rand(*shape, generator=g, device="cuda")


def _hidden(g, rows, d, dtype):
    """Hidden states: an offset, channels of uneven size, a few large ones."""
    channel = torch.exp(0.5 * _randn(g, d))
    channel[torch.randint(0, d, (max(1, d // 500),), generator=g, device="cuda")] *= 8.0
    return (_randn(g, rows, d) * channel + 0.3 * _randn(g, d)).to(dtype)


def _logits(g, T, V, dtype):
    """Logits with a few likely tokens per row among many unlikely ones, and every
    97th row's last eighth of the vocabulary ruled out."""
    x = 1.5 * _randn(g, T, V) - 2.0
    likely = torch.randint(0, V, (T, 12), generator=g, device="cuda")
    x.scatter_(1, likely, 10.0 + 2.0 * _randn(g, T, 12))
    x[::97, V - V // 8:] = float("-inf")
    return x.to(dtype)


def prepare(case, seed):
    c, g = case, _gen(seed)
    s = {"case": c}
    dtype = TYPES[c["type"]]
    if c["kind"] in ("block", "block_step"):
        rows, d = c["rows"], c["d"]
        s["b"], s["res"] = _hidden(g, rows, d, dtype), (2.0 * _hidden(g, rows, d, torch.float32)).to(dtype)
        weights = lambda: ((1.0 + 0.2 * _randn(g, d)).to(dtype), (0.1 * _randn(g, d)).to(dtype) if c["beta"] else None)
        s["gamma_after"], s["beta_after"] = weights() if c["after"] else (None, None)
        s["gamma"], s["beta"] = weights()
        s["gate"] = None
        if c["gate"] != "none":
            s["gate"] = (0.5 + 0.3 * (_randn(g, d) if c["gate"] == "vector" else _randn(g, rows, d))).to(dtype)
        if c["kind"] == "block_step":
            s["dy"] = (_randn(g, rows, d) + 0.1 * _randn(g, d)).to(dtype)
            s["dh"] = (0.5 * _randn(g, rows, d)).to(dtype)
    elif c["kind"] in ("product", "product_grad"):
        M, K, N = c["M"], c["K"], c["N"]
        s["x"] = _hidden(g, M, K, dtype)
        s["w"] = (_randn(g, N, K) / math.sqrt(K)).to(dtype)
        s["bias"] = (0.3 * _randn(g, N)).to(dtype) if c["bias"] else None
        s["residual"] = _hidden(g, M, N, dtype) if c["residual"] else None
        if c["kind"] == "product_grad":
            z = s["x"].float() @ s["w"].float().t()
            s["z"] = (z + s["bias"].float() if c["bias"] else z).to(dtype)
            s["dout"] = (_randn(g, M, N) + 0.1 * _randn(g, N)).to(dtype)
    else:
        T = c["T"]
        s["logits"] = _logits(g, T, c["V"], dtype)
        s["u"] = _rand(g, T)
        # every request has its own choices, around the case's
        s["temperature"] = c["temperature"] * (0.8 + 0.4 * _rand(g, T))
        s["top_k"] = s["top_p"] = s["min_p"] = None
        if c["top_k"] > 0:
            k = c["top_k"] * (0.8 + 0.4 * _rand(g, T))
            s["top_k"] = k.round().clamp(1, c["V"]).int()
        if c["top_p"] < 1.0:
            s["top_p"] = 1.0 - (1.0 - c["top_p"]) * (0.5 + _rand(g, T))
        if c["min_p"] > 0.0:
            s["min_p"] = c["min_p"] * (0.5 + _rand(g, T))
    return s


# ------------------------------------------------------- plain forms, 32 bits
def _plain_norm(x, gamma, beta, rms):
    if not rms:
        x = x - x.mean(dim=1, keepdim=True)
    rstd = torch.rsqrt(x.square().mean(dim=1, keepdim=True) + EPS)
    xh = x * rstd
    y = xh if gamma is None else xh * gamma.float()
    return (y if beta is None else y + beta.float()), xh, rstd


def _plain_norm_back(w, xh, rstd, rms):
    dx = w - xh * (w * xh).mean(dim=1, keepdim=True)
    return (dx if rms else dx - w.mean(dim=1, keepdim=True)) * rstd


def _plain_block(s):
    c, dtype = s["case"], TYPES[s["case"]["type"]]
    rms = c["norm"] == "rms"
    b = s["b"].float()
    n, bh, brstd = _plain_norm(b, s["gamma_after"], s["beta_after"], rms) if c["after"] else (b, b, None)
    gate = None if s["gate"] is None else s["gate"].float()
    h = c["rscale"] * s["res"].float() + (n if gate is None else gate * n)
    y, hh, hrstd = _plain_norm(h, s["gamma"], s["beta"], rms)
    out = [h.to(dtype), y.to(dtype)]
    if c["kind"] == "block":
        return out
    dy = s["dy"].float()
    dh = s["dh"].float() + _plain_norm_back(dy * s["gamma"].float(), hh, hrstd, rms)
    dn = dh if gate is None else dh * gate
    db = _plain_norm_back(dn * s["gamma_after"].float(), bh, brstd, rms) if c["after"] else dn
    out += [db, c["rscale"] * dh, (dy * hh).sum(dim=0)]
    if c["beta"]:
        out.append(dy.sum(dim=0))
    if gate is not None:
        out.append(dh * n if c["gate"] == "matrix" else (dh * n).sum(dim=0))
    if c["after"]:
        out.append((dn * bh).sum(dim=0))
        if c["beta"]:
            out.append(dn.sum(dim=0))
    return [t.to(dtype) for t in out]


def _tanh_inner(z):
    return math.sqrt(2.0 / math.pi) * (z + 0.044715 * z * z * z)


def _plain_act(z, act):
    if act == "relu":
        return torch.where(z > 0, z, 0.0)
    if act == "gelu":
        return 0.5 * z * (1.0 + torch.erf(z * math.sqrt(0.5)))
    if act == "gelu_tanh":
        return 0.5 * z * (1.0 + torch.tanh(_tanh_inner(z)))
    if act == "silu":
        return z / (1.0 + torch.exp(-z))
    return z


def _plain_act_slope(z, act):
    if act == "relu":
        return (z > 0).float()
    if act == "gelu":
        return 0.5 * (1.0 + torch.erf(z * math.sqrt(0.5))) + z * torch.exp(-0.5 * z * z) / math.sqrt(2.0 * math.pi)
    if act == "gelu_tanh":
        t = torch.tanh(_tanh_inner(z))
        return 0.5 * (1.0 + t) + 0.5 * z * (1.0 - t * t) * math.sqrt(2.0 / math.pi) * (1.0 + 3 * 0.044715 * z * z)
    if act == "silu":
        p = 1.0 / (1.0 + torch.exp(-z))
        return p * (1.0 + z * (1.0 - p))
    return torch.ones_like(z)


def _plain_product(s):
    c, dtype = s["case"], TYPES[s["case"]["type"]]
    x, w = s["x"].float(), s["w"].float()
    if c["kind"] == "product":
        z = x @ w.t()
        if s["bias"] is not None:
            z = z + s["bias"].float()
        y = _plain_act(z, c["act"])
        return (y if s["residual"] is None else y + s["residual"].float()).to(dtype)
    dz = s["dout"].float()
    if c["act"] != "none":
        dz = dz * _plain_act_slope(s["z"].float(), c["act"])
    out = [dz @ w, dz.t() @ x]
    if s["bias"] is not None:
        out.append(dz.sum(dim=0))
    return [t.to(dtype) for t in out]


def _plain_sample(s):
    """Kept tokens lie before a cut of the order (value descending, index
    ascending); the cuts and the draw compare sums, hence 64 bits."""
    x = s["logits"].float() + 0.0
    T, V = x.shape
    m = x.amax(dim=1, keepdim=True)
    w = torch.exp((x.double() - m.double()) / s["temperature"].double()[:, None])
    order = torch.sort(x, dim=1, descending=True, stable=True).indices
    ws = w.gather(1, order)
    kept = torch.ones_like(order, dtype=torch.bool)
    if s["top_k"] is not None:
        kept = torch.arange(V, device=x.device) < s["top_k"].long()[:, None]
    if s["top_p"] is not None:
        wk = torch.where(kept, ws, 0.0)
        before = torch.cumsum(wk, dim=1) - wk
        kept = kept & (before < s["top_p"].double()[:, None] * wk.sum(dim=1, keepdim=True))
    if s["min_p"] is not None:
        kept = kept & (ws >= s["min_p"].double()[:, None])
    w = torch.where(torch.zeros_like(kept).scatter_(1, order, kept), w, 0.0)
    total = w.sum(dim=1, keepdim=True)
    token = (torch.cumsum(w, dim=1) > s["u"].double()[:, None] * total).int().argmax(dim=1)
    logp = torch.log(w.gather(1, token[:, None]) / total)[:, 0]
    return token.int(), logp.float()


def _plain_run(s):
    kind = s["case"]["kind"]
    if kind in ("block", "block_step"):
        return _plain_block(s)
    if kind in ("product", "product_grad"):
        return _plain_product(s)
    return _plain_sample(s)


# ---------------------------------------------------------- the library's calls
def _empty(*shape, dtype=torch.float32):
    return torch.empty(*shape, dtype=dtype, device="cuda")


def _like(t):
    return None if t is None else torch.empty_like(t)


def _buffers(s, km):
    """The outputs and workspaces that a program keeps from call to call."""
    c = s["case"]
    dtype = TYPES[c["type"]]
    b = {}
    if c["kind"] in ("block", "block_step"):
        rows, d = c["rows"], c["d"]
        b["h"], b["y"] = torch.empty_like(s["b"]), torch.empty_like(s["b"])
        if c["kind"] == "block_step":
            b["stats"] = _empty(rows, 4)
            b["db"], b["dres"] = torch.empty_like(s["b"]), torch.empty_like(s["b"])
            b.update({"d" + k: _like(s[k]) for k in ("gamma", "beta", "gate", "gamma_after", "beta_after")})
            b["ws"] = _empty(km.kmp_block_norm_workspace_bytes(rows, d, dtype), dtype=torch.uint8)
    elif c["kind"] == "product":
        b["out"] = _empty(c["M"], c["N"], dtype=dtype)
    elif c["kind"] == "product_grad":
        b["dx"], b["dw"], b["dbias"] = torch.empty_like(s["x"]), torch.empty_like(s["w"]), _like(s["bias"])
        b["ws"] = _empty(km.kmp_dense_product_workspace_bytes(c["M"], c["N"], c["K"], dtype), dtype=torch.uint8)
    else:
        b["token"], b["logp"] = _empty(c["T"], dtype=torch.int32), _empty(c["T"])
        b["ws"] = _empty(km.kmp_sample_tokens_workspace_bytes(c["T"], c["V"]), dtype=torch.uint8)
    return b


def _own_run(s):
    from paper_2606_06742_amd import kmpath as km
    c = s["case"]
    if "buffers" not in s:
        s["buffers"] = _buffers(s, km)
    b = s["buffers"]
    if c["kind"] in ("block", "block_step"):
        form = dict(gate=s["gate"], gamma_after=s["gamma_after"], beta_after=s["beta_after"], gamma=s["gamma"],
                    rscale=c["rscale"], after=c["after"], rms=c["norm"] == "rms")
        km.kmp_block_norm(s["b"], s["res"], b["h"], b["y"], EPS, beta=s["beta"], stats=b.get("stats"), **form)
        if c["kind"] == "block":
            return b["h"], b["y"]
        km.kmp_block_norm_backward(s["dy"], s["dh"], s["b"], b["h"], b["stats"], b["db"], b["dres"],
                                   dgate=b["dgate"], dgamma_after=b["dgamma_after"], dbeta_after=b["dbeta_after"],
                                   dgamma=b["dgamma"], dbeta=b["dbeta"], workspace=b["ws"], **form)
        names = ("h", "y", "db", "dres", "dgamma", "dbeta", "dgate", "dgamma_after", "dbeta_after")
        return [b[k] for k in names if b[k] is not None]
    if c["kind"] == "product":
        km.kmp_dense_product(s["x"], s["w"], b["out"], bias=s["bias"], act=c["act"], residual=s["residual"])
        return b["out"]
    if c["kind"] == "product_grad":
        km.kmp_dense_product_backward(s["dout"], s["x"], s["w"], s["z"], b["dx"], b["dw"], b["dbias"], act=c["act"],
                                      workspace=b["ws"])
        return [b[k] for k in ("dx", "dw", "dbias") if b[k] is not None]
    km.kmp_sample_tokens(s["logits"], s["u"], b["token"], temperature=s["temperature"], top_k=s["top_k"],
                         top_p=s["top_p"], min_p=s["min_p"], logp=b["logp"], workspace=b["ws"])
    return b["token"], b["logp"]


def run(state):
    return _own_run(state) if own else _plain_run(state)


def work(case):
    c = case
    b = SIZE[c["type"]]
    if c["kind"] in ("block", "block_step"):
        n = c["rows"] * c["d"]
        vectors = (1 + c["beta"]) * (1 + c["after"]) + (c["gate"] == "vector")
        arrays, flops = 4 + (c["gate"] == "matrix"), (8 if c["after"] else 0) + 11
        if c["kind"] == "block":
            return {"bytes": b * (arrays * n + vectors * c["d"]), "flops": flops * n}
        return {"bytes": b * (2 * arrays * n + 2 * vectors * c["d"]), "flops": 3 * flops * n}
    if c["kind"] in ("product", "product_grad"):
        M, K, N = c["M"], c["K"], c["N"]
        if c["kind"] == "product":
            return {"bytes": b * (M * K + K * N + M * N * (1 + c["residual"]) + N * c["bias"]), "flops": 2 * M * K * N}
        # without an activation z is not read
        return {"bytes": b * (2 * M * K + 2 * K * N + M * N * (1 + (c["act"] != "none")) + N * c["bias"]),
                "flops": 4 * M * K * N}
    n = c["T"] * c["V"]
    requests = 4 + (c["top_k"] > 0) + (c["top_p"] < 1.0) + (c["min_p"] > 0.0)
    return {"bytes": b * n + 4 * c["T"] * requests, "flops": 5 * n}


# -------------------------------------------------------------- 64-bit results
def _exact_norm(x, gamma, beta, rms):
    first = 0.0 if rms else x.sum(dim=1, keepdim=True) / x.shape[1]
    second = (x * x).sum(dim=1, keepdim=True) / x.shape[1]
    y = (x - first) / torch.sqrt(second - first * first + EPS)
    if gamma is not None:
        y = y * gamma
    return y if beta is None else y + beta


def _exact_block(s):
    c = s["case"]
    rms = c["norm"] == "rms"
    names = [k for k in ("b", "res", "gamma", "beta", "gate", "gamma_after", "beta_after") if s[k] is not None]
    leaf = {k: s[k].double().requires_grad_(c["kind"] == "block_step") for k in names}
    at = leaf.get
    n = _exact_norm(leaf["b"], at("gamma_after"), at("beta_after"), rms) if c["after"] else leaf["b"]
    h = leaf["res"] * c["rscale"] + (n if s["gate"] is None else n * leaf["gate"])
    y = _exact_norm(h, leaf["gamma"], at("beta"), rms)
    if c["kind"] == "block":
        return [h, y]
    grads = torch.autograd.grad((h, y), [leaf[k] for k in names], (s["dh"].double(), s["dy"].double()))
    return [h.detach(), y.detach()] + list(grads)


_EXACT_ACT = {
    "none": lambda z: z * 1.0,
    "relu": torch.relu,
    "gelu": torch.nn.functional.gelu,
    "gelu_tanh": lambda z: torch.nn.functional.gelu(z, approximate="tanh"),
    "silu": torch.nn.functional.silu,
}


def _exact_product(s):
    c = s["case"]
    x, w = s["x"].double(), s["w"].double()
    if c["kind"] == "product":
        z = torch.matmul(x, w.t().contiguous())
        y = _EXACT_ACT[c["act"]](z if s["bias"] is None else z + s["bias"].double())
        return y if s["residual"] is None else s["residual"].double() + y
    z = s["z"].double().requires_grad_()
    dz = torch.autograd.grad(_EXACT_ACT[c["act"]](z), z, s["dout"].double())[0]
    out = [torch.matmul(dz, w), torch.matmul(dz.t().contiguous(), x)]
    return out + ([dz.sum(dim=0)] if s["bias"] is not None else [])


def _exact_row(s, t):
    """Token and log probability of row t by its sorted probabilities; the draw goes
    through the kept tokens sorted by index."""
    x = s["logits"][t].double()
    p = torch.softmax(x / s["temperature"][t].double(), dim=0)
    # descending values, ascending indices: the complemented order of a stable ascending sort
    index = x.numel() - 1 - torch.sort(x.flip(0) + 0.0, stable=True).indices.flip(0)
    if s["top_k"] is not None:
        index = index[:int(s["top_k"][t])]
    q = p[index]
    n = q.numel()
    if s["top_p"] is not None:
        sums = torch.cumsum(q, dim=0)
        n = min(n, 1 + int((sums < s["top_p"][t].double() * sums[-1]).sum()))
    if s["min_p"] is not None:
        n = min(n, int((q / q[0] >= s["min_p"][t].double()).sum()))
    index = torch.sort(index[:n]).values
    q = p[index]
    sums = torch.cumsum(q, dim=0)
    at = min(int((sums <= s["u"][t].double() * sums[-1]).sum()), n - 1)
    return index[at], torch.log(q[at]) - torch.log(sums[-1])


def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] in ("block", "block_step"):
        return _exact_block(s)
    if case["kind"] in ("product", "product_grad"):
        return _exact_product(s)
    rows = [_exact_row(s, t) for t in range(case["T"])]
    return torch.stack([r[0] for r in rows]).int(), torch.stack([r[1] for r in rows])

"""The operators at a language model's end in numpy, 64 bits, straight from
their definitions: layer norm and its gradients, rows in 8 bits and their
product, products with an activation, the norms around a block, log probabilities of tokens with entropy,
alternatives and gradient, tokens drawn from given random numbers."""
from __future__ import annotations

import numpy as np


def layer_norm(x, gamma, beta, eps):
    """(y, mean, rstd) of the rows of x."""
    x = np.asarray(x, dtype=np.float64)
    mean = x.mean(axis=1)
    rstd = 1.0 / np.sqrt(((x - mean[:, None]) ** 2).mean(axis=1) + eps)
    y = (x - mean[:, None]) * rstd[:, None]
    if gamma is not None:
        y = y * np.asarray(gamma, dtype=np.float64)
    if beta is not None:
        y = y + np.asarray(beta, dtype=np.float64)
    return y, mean, rstd


def layer_norm_backward(dy, x, gamma, mean, rstd):
    """(dx, dgamma, dbeta) at the given mean and rstd."""
    dy, x = np.asarray(dy, dtype=np.float64), np.asarray(x, dtype=np.float64)
    xh = (x - mean[:, None]) * rstd[:, None]
    w = dy if gamma is None else dy * np.asarray(gamma, dtype=np.float64)
    dx = rstd[:, None] * (w - w.mean(axis=1)[:, None] - xh * (w * xh).mean(axis=1)[:, None])
    return dx, (dy * xh).sum(axis=0), dy.sum(axis=0)


def block_norm(b, res, gamma_after, beta_after, gate, gamma, beta, eps, rscale=1.0, after=True, rms=False):
    """(h, y, stats): h = rscale res + gate N(b), y = N(h), stats (rows, 4) the mean
    and factor of either norm (0 and 1 without `after`)."""
    def norm(x, g, c):
        mean = np.zeros(len(x)) if rms else x.mean(axis=1)
        r = 1.0 / np.sqrt(((x - mean[:, None]) ** 2).mean(axis=1) + eps)
        y = (x - mean[:, None]) * r[:, None]
        y = y if g is None else y * np.asarray(g, np.float64)
        return (y if c is None else y + np.asarray(c, np.float64)), mean, r

    b = np.asarray(b, np.float64)
    n, m1, r1 = norm(b, gamma_after, beta_after) if after else (b, np.zeros(len(b)), np.ones(len(b)))
    h = n if gate is None else np.asarray(gate, np.float64) * n
    if res is not None:
        h = rscale * np.asarray(res, np.float64) + h
    y, m2, r2 = norm(h, gamma, beta)
    return h, y, np.stack([m1, r1, m2, r2], axis=1)


def block_norm_backward(dy, dh, b, h, stats, gamma_after, beta_after, gate, gamma, rscale=1.0, after=True, rms=False):
    """dict of db, dres, dgate (per row and element), dgamma_after, dbeta_after,
    dgamma, dbeta at the given h and stats; s, t as intermediate results."""
    f = lambda a, none: none if a is None else np.asarray(a, np.float64)
    b = f(b, None)
    m1, r1, m2, r2 = (stats[:, i:i + 1].astype(np.float64) for i in range(4))
    ga, ca, g0, g2 = f(gamma_after, 1.0), f(beta_after, 0.0), f(gate, 1.0), f(gamma, 1.0)

    def back(w, xh, r):
        dx = w - xh * (w * xh).mean(axis=1, keepdims=True)
        return r * (dx if rms else dx - w.mean(axis=1, keepdims=True))

    s = f(dh, np.zeros_like(b))
    out = dict(dgamma=np.zeros(b.shape[1]), dbeta=np.zeros(b.shape[1]))
    if dy is not None:
        xh2 = (np.asarray(h, np.float64) - m2) * r2
        s = s + back(f(dy, None) * g2, xh2, r2)
        out.update(dgamma=(dy * xh2).sum(axis=0), dbeta=np.asarray(dy, np.float64).sum(axis=0))
    t = s * g0
    xh1 = (b - m1) * r1 if after else b
    n = xh1 * ga + ca if after else b
    out.update(s=s, t=t, dres=rscale * s, dgate=s * n, db=back(t * ga, xh1, r1) if after else t,
               dgamma_after=(t * xh1).sum(axis=0), dbeta_after=t.sum(axis=0))
    return out


def quantize_rows(x):
    """(q, scale): the definition in 32-bit arithmetic, every operation rounded
    once, as the result is a whole number that depends on those roundings."""
    x = np.asarray(x, dtype=np.float32)
    with np.errstate(all="ignore"):
        a = np.abs(x).max(axis=1)                  # NaN where a row has one
        lift = np.where(a < np.float32(2.0 ** -100), np.float32(2.0 ** 100), np.float32(1.0)).astype(np.float32)
        good = a < np.inf
        factor = np.where(good & (a > 0), np.float32(1.0) / (a * lift) * np.float32(127.0), np.float32(0.0)).astype(np.float32)
        q = np.rint((x * lift[:, None]) * factor[:, None])
        q = np.where((factor > 0)[:, None], np.clip(q, -127, 127), 0)
        scale = np.where(good, a / np.float32(127.0), np.float32(np.nan)).astype(np.float32)
    return np.nan_to_num(q).astype(np.int8), scale


def quantized_product(xq, xscale, wq, wscale, bias=None):
    y = np.asarray(xq, np.float64) @ np.asarray(wq, np.float64).T        # whole numbers below 2^53: exact
    y = y * np.asarray(xscale, np.float64)[:, None] * np.asarray(wscale, np.float64)[None, :]
    return y if bias is None else y + np.asarray(bias, np.float64)


def activation(z, act):
    """(act(z), act'(z))."""
    from scipy.special import erf
    z = np.asarray(z, np.float64)
    if act == "relu":
        return np.maximum(z, 0.0), (z > 0).astype(np.float64)
    if act == "gelu":
        p = 0.5 * (1.0 + erf(z / np.sqrt(2.0)))
        return z * p, p + z * np.exp(-0.5 * z * z) / np.sqrt(2.0 * np.pi)
    if act == "gelu_tanh":
        c = np.sqrt(2.0 / np.pi)
        t = np.tanh(c * (z + 0.044715 * z ** 3))
        return 0.5 * z * (1.0 + t), 0.5 * (1.0 + t) + 0.5 * z * (1.0 - t * t) * c * (1.0 + 3 * 0.044715 * z * z)
    if act == "silu":
        with np.errstate(over="ignore"):
            p = 1.0 / (1.0 + np.exp(-z))
        return z * p, p * (1.0 + z * (1.0 - p))
    return z, np.ones_like(z)


def dense_product(x, w, bias=None, act="none", residual=None):
    """(out, z): out = act(z) + residual, z = x w' + bias."""
    z = np.asarray(x, np.float64) @ np.asarray(w, np.float64).T
    if bias is not None:
        z = z + np.asarray(bias, np.float64)
    y = activation(z, act)[0]
    return (y if residual is None else y + np.asarray(residual, np.float64)), z


def dense_product_backward(dout, x, w, z, act="none"):
    """(dx, dw, dbias, dz) at the given z."""
    dz = np.asarray(dout, np.float64)
    if act != "none":
        dz = dz * activation(z, act)[1]
    return dz @ np.asarray(w, np.float64), dz.T @ np.asarray(x, np.float64), dz.sum(axis=0), dz


def token_logprobs(x, tokens, top=0):
    """dict of logp, entropy, stats (the maximum, the log of the sum of exp(x -
    maximum)), lse (their sum), top_id, top_logp for logits x (T, V)."""
    x = np.asarray(x, dtype=np.float64)
    T, V = x.shape
    out = dict(logp=np.zeros(T), entropy=np.zeros(T), lse=np.zeros(T), stats=np.zeros((T, 2)),
               top_id=np.zeros((T, top), np.int32), top_logp=np.zeros((T, top)))
    for t in range(T):
        r = x[t]
        # NaN above all, then values descending, equal ones by index
        order = np.lexsort((np.arange(V), -np.where(np.isnan(r), 0.0, r), ~np.isnan(r)))[:top]
        out["top_id"][t] = order
        if np.all(r == -np.inf):
            m = logs = lse = -np.inf
            H, lp = 0.0, np.full(V, -np.inf)
        elif np.isnan(r).any() or np.any(r == np.inf):
            m = logs = lse = H = np.nan
            lp = np.full(V, np.nan)
        else:
            m, logs = r.max(), np.log(np.exp(r - r.max()).sum())
            lse = m + logs
            lp = (r - m) - logs                    # exact to rounding at any size of m
            live = r > -np.inf
            H = -(np.exp(lp[live]) * lp[live]).sum()
        out["lse"][t], out["entropy"][t], out["top_logp"][t] = lse, H, lp[order]
        out["stats"][t] = m, logs
        k = -1 if tokens is None else int(tokens[t])
        out["logp"][t] = 0.0 if k < 0 else np.nan if k >= V else lp[k]
    return out


def token_logprobs_backward(x, tokens, stats, dlogp=None, entropy=None, dentropy=None):
    """Gradient of sum dlogp logp + dentropy entropy at the given stats, entropy."""
    x = np.asarray(x, dtype=np.float64)
    T, V = x.shape
    dx = np.zeros((T, V))
    for t in range(T):
        k = -1 if tokens is None or dlogp is None else int(tokens[t])
        if k >= V or np.isnan(stats[t]).any():
            dx[t] = np.nan
            continue
        if stats[t][0] == -np.inf:
            continue
        live = x[t] > -np.inf
        lp = (x[t][live] - stats[t][0]) - stats[t][1]
        p = np.exp(lp)
        if dentropy is not None:
            dx[t, live] -= dentropy[t] * p * (lp + entropy[t])
        if k >= 0:
            dx[t, live] -= dlogp[t] * p
            dx[t, k] += dlogp[t]
    return dx


def sample_tokens(x, u, temperature=None, top_k=None, top_p=None, min_p=None):
    """(tokens, logp, margin): tokens drawn from the rows of x as defined. margin is how
    near, relative to the sums, a comparison came that decides the token."""
    x = np.asarray(x, dtype=np.float64)
    T, V = x.shape
    tokens, logp, margin = np.full(T, -1, np.int64), np.full(T, np.nan), np.full(T, np.inf)
    at = lambda a, t, none: none if a is None else float(a[t])
    for t in range(T):
        r = x[t]
        c = at(temperature, t, 1.0), at(top_p, t, 1.0), at(min_p, t, 0.0), float(u[t])
        k = V if top_k is None or top_k[t] <= 0 else min(int(top_k[t]), V)
        if np.isnan(c).any() or np.isnan(r).any() or np.any(r == np.inf):
            continue
        if np.all(r == -np.inf):
            logp[t] = -np.inf
            continue
        order = np.lexsort((np.arange(V), -r))
        if c[0] <= 0:
            tokens[t], logp[t] = order[0], 0.0
            continue
        w = np.zeros(V)
        live = r > -np.inf
        with np.errstate(under="ignore"):
            w[live] = np.exp((r[live] - r.max()) / c[0])
        order = order[:k]
        if c[1] < 1:
            sums = np.cumsum(w[order].astype(np.longdouble))
            reach = c[1] * sums[-1]
            n = int(np.searchsorted(sums, reach, side="left")) + 1 if c[1] > 0 else 1
            if 0 < c[1]:
                margin[t] = min(margin[t], float(np.abs(sums - reach).min() / sums[-1]))
            order = order[:min(n, len(order))]
        if c[2] > 0:
            floor = min(c[2], 1.0)
            near = np.abs(w[order] / floor - 1)
            near = near[w[order] != floor]
            margin[t] = min(margin[t], float(near.min()) if near.size else np.inf)
            order = order[w[order] >= floor]
        kept = np.sort(order)
        sums = np.cumsum(w[kept].astype(np.longdouble))
        goal = min(max(c[3], 0.0), 1.0) * sums[-1]
        over = np.flatnonzero(sums > goal)
        i = int(over[0]) if over.size else int(np.flatnonzero(w[kept] > 0)[-1])
        if goal > 0:
            margin[t] = min(margin[t], float(np.abs(sums - goal)[:-1].min() / sums[-1]) if len(sums) > 1 else np.inf)
        tokens[t], logp[t] = kept[i], np.log(w[kept[i]]) - float(np.log(sums[-1]))
    return tokens, logp, margin

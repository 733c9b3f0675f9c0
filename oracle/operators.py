"""The operators at a language model's end in numpy, 64 bits, straight from
their definitions: layer norm and its gradients, rows in 8 bits and their
product, log probabilities of tokens with entropy, alternatives and gradient."""
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

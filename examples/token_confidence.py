"""Which answers of a language model are right? A kernel machine on what the
model's end says about them.

A model's last hidden states go through its layer norm, an 8-bit vocabulary head
and the log probabilities of the answers' tokens. First the norm's weights are
trained for a few steps on answers that are known (the gradients go back through
the same operators; the rounding to 8 bits is passed straight through). Then every
answer's log probability, entropy and lead over its alternatives become features,
and the cross-validated path of a kernel logistic regression learns from them
whether an answer is right.

The hidden states are synthetic: each is the direction of the answer the model
means, more or less blurred, and the model is right where it means the true one.

    python examples/token_confidence.py [--answers N] [--width K] [--vocabulary V]
"""
from __future__ import annotations

import argparse
import os
import sys

import numpy as np
import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2606_06742_amd import kmpath as km  # noqa: E402

EPS = 1e-5


class Tail:
    """Norm, 8-bit head and token log probabilities, with their buffers, for T
    hidden states of width K and V tokens."""

    def __init__(self, head, T, top):
        dev, (V, K) = head.device, head.shape
        self.head, self.T, self.top = head, T, top
        empty = lambda *s, dtype=torch.float32: torch.empty(*s, dtype=dtype, device=dev)
        # the head in 8 bits, once: rows at multiples of 64 bytes are read fastest
        pitch = (K + 63) // 64 * 64
        self.wq, self.wscale = empty(V, pitch, dtype=torch.int8)[:, :K], empty(V)
        km.kmp_quantize_rows(head, self.wq, self.wscale)
        self.gamma, self.beta = torch.ones(K, device=dev), torch.zeros(K, device=dev)
        self.q, self.qscale = empty(T, pitch, dtype=torch.int8)[:, :K], empty(T)
        self.mean, self.rstd = empty(T), empty(T)
        self.logits = empty(T, V)
        self.logp, self.entropy, self.stats = empty(T), empty(T), empty(T, 2)
        self.top_id, self.top_logp = empty(T, top, dtype=torch.int32), empty(T, top)
        self.dgamma, self.dbeta = torch.empty_like(self.gamma), torch.empty_like(self.beta)
        self.ws = empty(max(km.kmp_token_logprobs_workspace_bytes(T, V, top),
                            km.kmp_layer_norm_workspace_bytes(T, K, torch.bfloat16)), dtype=torch.uint8)

    def forward(self, hidden, tokens):
        """Log probability and entropy of each token, and the alternatives."""
        km.kmp_layer_norm(hidden, self.gamma, self.beta, EPS, self.q, mean=self.mean, rstd=self.rstd,
                          scale=self.qscale)
        km.kmp_quantized_product(self.q, self.qscale, self.wq, self.wscale, self.logits)
        km.kmp_token_logprobs(self.logits, tokens, self.logp, entropy=self.entropy, stats=self.stats,
                              top_id=self.top_id, top_logp=self.top_logp, workspace=self.ws)
        return self.logp

    def train_step(self, hidden, tokens, rate):
        """One step on the norm's weights; the mean loss before it."""
        loss = -self.forward(hidden, tokens).mean()
        dlogp = torch.full((self.T,), -1.0 / self.T, device=hidden.device)
        km.kmp_token_logprobs_backward(self.logits, tokens, self.stats, dlogp, self.logits)
        dy = (self.logits @ self.head).to(hidden.dtype)
        km.kmp_layer_norm_backward(dy, hidden, self.gamma, self.mean, self.rstd, None, self.dgamma, self.dbeta,
                                   self.ws)
        self.gamma -= rate * self.dgamma
        self.beta -= rate * self.dbeta
        return float(loss)


def answers(n, K, V, seed, device):
    """head (V, K), hidden states (n, K), true tokens (n), 1 where right."""
    g = torch.Generator(device=device)
    g.manual_seed(seed)
    head = torch.randn(V, K, generator=g, device=device) / K ** 0.5
    true = torch.randint(0, V, (n,), generator=g, device=device)
    other = torch.randint(0, V, (n,), generator=g, device=device)
    sure = torch.rand(n, generator=g, device=device)                 # how clearly the model means its answer
    right = torch.rand(n, generator=g, device=device) < 0.2 + 0.75 * sure
    means = torch.where(right, true, other)
    hidden = head[means] * K ** 0.5 * (0.25 + sure)[:, None] + 2.0 * torch.randn(n, K, generator=g, device=device)
    return head, (hidden * 0.5 + 0.1).to(torch.bfloat16), means, torch.where(right, 1.0, -1.0).double()


def run(n=1200, K=512, V=8000, steps=5, seed=1, device="cuda", say=print):
    head, hidden, means, y = answers(n, K, V, seed, device)
    tail = Tail(head, n, top=5)
    losses = [tail.train_step(hidden, means, rate=20.0) for _ in range(steps)]
    tail.forward(hidden, means)
    losses.append(float(-tail.logp.mean()))
    say("loss of the known answers, by steps on the norm: " + " ".join("%.3f" % v for v in losses))

    lead = tail.top_logp[:, 0] - tail.top_logp[:, 1:].mean(dim=1)
    X = torch.stack([tail.top_logp[:, 0], tail.entropy, lead], dim=1).double()
    X = ((X - X.mean(dim=0)) / X.std(dim=0)).contiguous()
    sigma = float(torch.pdist(X[:500]).median())
    lambdas = 10.0 ** np.linspace(-4.0, 0.0, 9)
    folds = km.kmp_make_folds(n, 5, seed)
    fit = km.fit_path(X, y, "logistic", [sigma], lambdas, folds, 5)
    best = int(fit["selected"][0, 0])
    wrong = float(fit["cv_err"][0, 0, :, best].sum()) / n
    base = float((y < 0).double().mean())
    say("right answers %.1f %%; cross-validated error of telling them apart %.1f %% at lambda %.1e"
        % (100 * (1 - base), 100 * wrong, lambdas[best]))
    return {"losses": losses, "error": wrong, "base": min(base, 1 - base)}


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--answers", type=int, default=1200)
    ap.add_argument("--width", type=int, default=512)
    ap.add_argument("--vocabulary", type=int, default=8000)
    a = ap.parse_args()
    run(a.answers, a.width, a.vocabulary)

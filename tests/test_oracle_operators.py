"""The plain operators of oracle/operators.py against torch's own definitions
in 64 bits on the CPU and against central differences."""
import numpy as np
import pytest
import torch

from oracle import operators as OO


def test_layer_norm_and_gradients_against_autograd():
    rng = np.random.default_rng(1)
    x, g, b, dy = rng.standard_normal((5, 7)), rng.standard_normal(7), rng.standard_normal(7), rng.standard_normal((5, 7))
    y, mean, rstd = OO.layer_norm(x, g, b, 1e-5)
    tx, tg, tb = (torch.tensor(v, requires_grad=True) for v in (x, g, b))
    ty = torch.nn.functional.layer_norm(tx, (7,), tg, tb, 1e-5)
    assert np.allclose(y, ty.detach().numpy(), rtol=1e-13, atol=1e-13)
    want = torch.autograd.grad(ty, (tx, tg, tb), torch.tensor(dy))
    for a, w in zip(OO.layer_norm_backward(dy, x, g, mean, rstd), want):
        assert np.allclose(a, w.numpy(), rtol=1e-11, atol=1e-12)


def test_layer_norm_gradient_against_differences():
    rng = np.random.default_rng(2)
    x, g, b, dy = rng.standard_normal((2, 9)), rng.standard_normal(9), rng.standard_normal(9), rng.standard_normal((2, 9))
    _, mean, rstd = OO.layer_norm(x, g, b, 1e-3)
    dx, dg, _ = OO.layer_norm_backward(dy, x, g, mean, rstd)
    h = 1e-5                                       # error h^2 times a third derivative of order 10
    for i in np.ndindex(*x.shape):
        e = np.zeros_like(x)
        e[i] = h
        d = ((OO.layer_norm(x + e, g, b, 1e-3)[0] - OO.layer_norm(x - e, g, b, 1e-3)[0]) * dy).sum() / (2 * h)
        assert abs(d - dx[i]) < 1e-7
    for j in range(9):
        e = np.zeros_like(g)
        e[j] = h
        d = ((OO.layer_norm(x, g + e, b, 1e-3)[0] - OO.layer_norm(x, g - e, b, 1e-3)[0]) * dy).sum() / (2 * h)
        assert abs(d - dg[j]) < 1e-7


def test_quantize_rows_definition():
    x = np.array([[1.0, -2.0, 0.5], [0.0, 0.0, 0.0], [np.inf, 1.0, 2.0], [np.nan, 1.0, 2.0], [1e-42, 0.0, -2e-42]])
    q, s = OO.quantize_rows(x)
    assert q.tolist() == [[64, -127, 32], [0, 0, 0], [0, 0, 0], [0, 0, 0], [64, 0, -127]]
    assert s[0] == np.float32(2.0) / np.float32(127.0) and s[1] == 0 and np.isnan(s[2]) and np.isnan(s[3])


@pytest.mark.parametrize("mask", [False, True])
def test_token_logprobs_against_autograd(mask):
    rng = np.random.default_rng(3)
    x = rng.standard_normal((6, 11))
    if mask:
        x[:, 3] = -np.inf
    tok = np.array([0, 10, -1, 5, 4, 2])
    g, h = rng.standard_normal(6), rng.standard_normal(6)
    o = OO.token_logprobs(x, tok, top=4)
    tx = torch.tensor(x, requires_grad=True)
    lp = torch.log_softmax(tx, dim=1)
    H = -(lp.exp() * lp.masked_fill(lp == -np.inf, 0.0)).sum(dim=1)
    at = torch.stack([lp[t, k] if k >= 0 else lp.new_zeros(()) for t, k in enumerate(tok)])
    assert np.allclose(o["logp"], at.detach().numpy(), atol=1e-13) and np.allclose(o["entropy"], H.detach().numpy(), atol=1e-13)
    vals, ids = torch.sort(lp.detach(), dim=1, descending=True, stable=True)
    assert np.array_equal(o["top_id"], ids[:, :4].numpy()) and np.allclose(o["top_logp"], vals[:, :4].numpy(), atol=1e-13)
    want = torch.autograd.grad((at * torch.tensor(g)).sum() + (H * torch.tensor(h)).sum(), tx)[0].numpy()
    got = OO.token_logprobs_backward(x, tok, o["stats"], g, o["entropy"], h)
    assert np.allclose(got, want, atol=1e-13)


def test_token_logprobs_gradient_against_differences():
    rng = np.random.default_rng(4)
    x, tok, g, h = rng.standard_normal((2, 5)), np.array([1, 4]), rng.standard_normal(2), rng.standard_normal(2)
    o = OO.token_logprobs(x, tok)
    dx = OO.token_logprobs_backward(x, tok, o["stats"], g, o["entropy"], h)

    def f(z):
        r = OO.token_logprobs(z, tok)
        return (g * r["logp"]).sum() + (h * r["entropy"]).sum()

    for i in np.ndindex(*x.shape):
        e = np.zeros_like(x)
        e[i] = 1e-5
        assert abs((f(x + e) - f(x - e)) / 2e-5 - dx[i]) < 1e-8


def test_token_logprobs_edges():
    x = np.array([[-np.inf] * 4, [np.nan, 1.0, 2.0, 0.0], [np.inf, 1.0, -np.inf, 0.0], [2.0, 2.0, -0.0, 0.0]])
    o = OO.token_logprobs(x, np.array([1, 1, 1, 7]), top=4)
    assert o["lse"][0] == -np.inf and o["logp"][0] == -np.inf and o["entropy"][0] == 0
    assert np.isnan(o["logp"][1:]).all() and np.isnan(o["entropy"][1:3]).all()
    assert o["top_id"].tolist() == [[0, 1, 2, 3], [0, 2, 1, 3], [0, 1, 3, 2], [0, 1, 2, 3]]
    dx = OO.token_logprobs_backward(x, np.array([1, 1, 1, 7]), o["stats"], np.ones(4))
    assert (dx[0] == 0).all() and np.isnan(dx[1:]).all()

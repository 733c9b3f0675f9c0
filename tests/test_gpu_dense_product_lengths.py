"""Products of every number of slices of k, and of a few tokens with more output channels than
one launch has threads for, in whole numbers, which every form sums exactly."""
import numpy as np
import pytest

from tests.gpu_common import announce, device
from tests.test_gpu_operators import _dtype

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("xt,M,N,K", [("bf16", 1, 2 ** 28 - 16, 3), ("bf16", 1, 2 ** 28 - 15, 3), ("f16", 4, 2 ** 28 + 33, 2),
                                      ("f32", 2, 2 ** 28 + 1, 4), ("bf16", 1, 2 ** 29, 8)])
def test_channels_beyond_a_launch(xt, M, N, K):
    import torch
    from paper_2606_06742_amd import kmpath as km
    announce(f"dense product {xt} {M} x {N} x {K}")
    t = _dtype(xt)
    x = (torch.arange(M * K, device=device()) % 5 - 2).reshape(M, K).to(t)
    w = torch.empty(N, K, dtype=t, device=device())
    want = torch.zeros(M, N, dtype=t, device=device())
    n = torch.arange(N, device=device(), dtype=torch.int32)
    for k in range(K):
        w[:, k] = ((n * (k + 1)) % 13 - 6).to(t)
        for m in range(M):
            want[m] += x[m, k] * w[:, k]
    out = torch.full((M, N), float("nan"), dtype=t, device=device())
    km.kmp_dense_product(x, w, out)
    torch.cuda.synchronize()
    assert torch.equal(out, want)


@pytest.mark.parametrize("xt", ["f32", "bf16"])
@pytest.mark.parametrize("M,N", [(2048, 2048), (3000, 2900), (4096, 4096)])
def test_every_number_of_slices(xt, M, N):
    """One slice of 128 bytes up to eleven, with and without a rest, in each of the larger
    forms; the gradients sum over as many tokens, with both operands taken as they are."""
    import torch
    from paper_2606_06742_amd import kmpath as km
    t, per = _dtype(xt), 128 // _dtype(xt).itemsize
    rng = np.random.default_rng(M)
    at = lambda n, to: torch.as_tensor(rng.integers(0, to, n), device=device())
    rows = lambda n: torch.arange(n, device=device())
    for slices in range(12):
        for rest in (0, 8):
            K = slices * per + rest
            if K == 0:
                continue
            announce(f"dense product, {slices} slices, {xt} {M} x {N} x {K}")
            x, w = torch.zeros(M, K, dtype=t, device=device()), torch.zeros(N, K, dtype=t, device=device())
            i, j = at(M, K), at(N, K)
            x[rows(M), i] = 1
            w[rows(N), j] = 1
            out = torch.full((M, N), float("nan"), dtype=t, device=device())
            km.kmp_dense_product(x, w, out)
            assert torch.equal(out, (i[:, None] == j[None, :]).to(t))
            # dw (M x N here) = dz' x over K tokens, each with one channel
            dz, y = torch.zeros(K, M, dtype=t, device=device()), torch.zeros(K, N, dtype=t, device=device())
            c = at(K, M)
            dz[rows(K), c] = 1
            y[:] = torch.as_tensor(rng.integers(-3, 4, (K, N)), device=device()).to(t)
            dw = torch.full((M, N), float("nan"), dtype=t, device=device())
            ws = torch.full((km.kmp_dense_product_workspace_bytes(K, M, N, t),), 255, dtype=torch.uint8, device=device())
            km.kmp_dense_product_backward(dz, y, None, None, None, dw, None, workspace=ws)
            assert torch.equal(dw.float(), torch.zeros(M, N, device=device()).index_add_(0, c, y.float()))


def test_every_number_of_slices_in_8_bits():
    import torch
    from paper_2606_06742_amd import kmpath as km
    rng = np.random.default_rng(3)
    for M, N in ((2048, 2048), (3000, 2900), (4096, 4096)):
        for K in (16, 128, 144, 256, 272, 384, 400, 512, 528, 640, 656, 768, 1152, 1168):
            announce(f"8-bit product {M} x {N} x {K}")
            x, w = (torch.as_tensor(rng.integers(-9, 10, (n, K)), dtype=torch.int8, device=device()) for n in (M, N))
            one = torch.ones(max(M, N), device=device())
            out = torch.full((M, N), float("nan"), device=device())
            km.kmp_quantized_product(x, one[:M], w, one[:N], out)
            assert torch.equal(out, x.float() @ w.float().T)    # (whole numbers below 2^24)


@pytest.mark.parametrize("xt", ["f32", "bf16"])
def test_bias_of_more_channels_than_workgroups(xt):
    """The sums over the tokens take up to 2^20 workgroups, each then more than one tile."""
    import torch
    from paper_2606_06742_amd import kmpath as km
    M, N, t = 9, 2 ** 27 + 77, _dtype(xt)
    announce(f"dense product, bias of {M} x {N} {xt}")
    n = torch.arange(N, device=device(), dtype=torch.int32)
    dout = torch.empty(M, N, dtype=t, device=device())
    for m in range(M):
        dout[m] = ((n + m * 5) % 11 - 5).to(t)
    db = torch.full((N,), float("nan"), device=device())
    ws = torch.empty(km.kmp_dense_product_workspace_bytes(M, N, 0, t), dtype=torch.uint8, device=device())
    km.kmp_dense_product_backward(dout, None, None, None, None, None, db, workspace=ws)
    assert torch.equal(db, dout.float().sum(dim=0))


def test_gradients_of_a_few_tokens_in_long_rows():
    """8 tokens of 2^26 elements and one channel: the runs' join takes up to 2^20 workgroups,
    each then more than one part."""
    import torch
    from paper_2606_06742_amd import kmpath as km
    M, N, K, t = 8, 1, 2 ** 26 + 3, torch.bfloat16
    announce(f"dense product, gradients of {M} x {N} x {K}")
    k = torch.arange(K, device=device(), dtype=torch.int32)
    dout = (torch.arange(M, device=device()) - 3).reshape(M, N).to(t)
    w, x = (k % 13 - 6).to(t).reshape(N, K), torch.empty(M, K, dtype=t, device=device())
    for m in range(M):
        x[m] = ((k + m) % 7 - 3).to(t)
    dx, dw = torch.full((M, K), float("nan"), dtype=t, device=device()), torch.full((N, K), float("nan"), dtype=t, device=device())
    ws = torch.empty(km.kmp_dense_product_workspace_bytes(M, N, K, t), dtype=torch.uint8, device=device())
    km.kmp_dense_product_backward(dout, x, w, None, dx, dw, None, workspace=ws)
    assert torch.equal(dx, dout * w)
    assert torch.equal(dw[0], (dout.float() * x.float()).sum(dim=0).to(t))     # (whole numbers up to 84)

"""Products of a few tokens with more output channels than one launch has threads for, in
whole numbers, which every form sums exactly."""
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

"""Workspace sizes on the host: a workspace of a program's largest call serves its smaller
ones, also around every border at which the library changes how it divides the work."""
import torch

from tests.test_operators_abi import km  # noqa: F401


def _does_not_fall(sizes):
    return min(sizes) > 0 and all(a <= b for a, b in zip(sizes, sizes[1:]))


def _around(*borders):
    return sorted({max(1, b + e) for b in borders for e in (-1, 0, 1)})


def test_sampling(km):  # noqa: F811
    size = km.kmp_sample_tokens_workspace_bytes
    lengths = _around(*(1 << i for i in range(31)), *(i << 20 for i in range(1, 40)), 1500000, 2 ** 31 - 2,
                      *(i << 14 for i in range(1, 70)))
    for T in (1, 2, 255, 256, 257, 70000, 2 ** 31 - 1):
        assert _does_not_fall([size(T, V) for V in lengths]), T
    for V in lengths:
        assert _does_not_fall([size(T, V) for T in (0, 1, 2, 256, 257, 65536, 2 ** 31 - 1)]), V


def test_norms_and_products(km):  # noqa: F811
    counts = _around(8, 16, 64, 256, 512, 1024, 2048, 4096, 8192, 16384, 1 << 20)
    for dtype in (torch.float32, torch.bfloat16):
        for n in counts:
            assert _does_not_fall([km.kmp_block_norm_workspace_bytes(n, d, dtype) for d in counts])
            assert _does_not_fall([km.kmp_block_norm_workspace_bytes(r, n, dtype) for r in counts])
            for m in (1, 8, 9, 300, 4096):
                assert _does_not_fall([km.kmp_dense_product_workspace_bytes(v, n, m, dtype) for v in counts])
                assert _does_not_fall([km.kmp_dense_product_workspace_bytes(m, v, n, dtype) for v in counts])
                assert _does_not_fall([km.kmp_dense_product_workspace_bytes(n, m, v, dtype) for v in counts])

"""kmp_sample_tokens on the host: refusals and workspace sizes; the oracle's draws
against probabilities written out by hand."""
import numpy as np
import torch

from oracle import operators as OO
from tests.test_operators_abi import P, km  # noqa: F401


def test_refusals(km):  # noqa: F811
    need = km.kmp_sample_tokens_workspace_bytes(4, 100)
    assert need >= 256

    def call(t=1, x=P, T=4, V=100, ld=100, u=P, bits=32, tok=P, ws=P, n=need):
        return km.lib().kmp_sample_tokens(None, t, x, T, V, ld, u, P, P, P, P, bits, tok, P, ws, n)

    for b in (dict(t=0), dict(t=4), dict(x=None), dict(T=-1), dict(T=1 << 31), dict(V=0), dict(V=1 << 31, ld=1 << 31), dict(ld=99),
              dict(ld=(1 << 40) + 1), dict(u=None), dict(bits=16), dict(tok=None)):
        assert call(**b) == km.KMP_EINVAL, b
        assert "kmp_sample_tokens" in km.kmp_strerror(km.KMP_EINVAL)
    assert call(ws=None) == km.KMP_EWORKSPACE and call(n=need - 1) == km.KMP_EWORKSPACE and call(ws=P + 8) == km.KMP_EWORKSPACE
    assert call(T=0, x=None, u=None, tok=None, ws=None) == km.KMP_OK
    for a in ((-1, 5), (1, 0), (1 << 31, 5), (5, 1 << 31)):
        assert km.kmp_sample_tokens_workspace_bytes(*a) == 0
    import pytest
    with pytest.raises(km.KmpError, match="logits must be a 2-D device tensor"):
        km.kmp_sample_tokens(torch.zeros(2, 3), None, None)


def test_workspace_does_not_fall(km):  # noqa: F811
    """A workspace of a program's largest call serves its smaller ones."""
    size = km.kmp_sample_tokens_workspace_bytes
    rows = (0, 1, 2, 3, 7, 8, 16, 63, 64, 65, 128, 255, 256, 257, 1000, 100000, 2 ** 31 - 1)
    for V in (1, 1000, 8192, 32000, 65536, 128000, 1 << 20, 2 ** 31 - 1):
        sizes = [size(T, V) for T in rows]
        assert sizes == sorted(sizes), V
    for T in rows:
        sizes = [size(T, V) for V in (1, 1000, 4096, 4097, 8192, 16385, 32000, 65536, 65537, 128000, 262145, 1 << 25, 2 ** 31 - 1)]
        assert sizes == sorted(sizes), T


def test_oracle_by_hand():
    """Four tokens of probabilities 0.1, 0.4, 0.2, 0.3."""
    x = np.log(np.array([[0.1, 0.4, 0.2, 0.3]]))
    draw = lambda u, **k: int(OO.sample_tokens(x, [u], **{n: [v] for n, v in k.items()})[0][0])
    assert [draw(u) for u in (0.05, 0.15, 0.45, 0.55, 0.65, 0.75, 0.99)] == [0, 1, 1, 2, 2, 3, 3]
    assert [draw(u, top_k=2) for u in (0.5, 0.6)] == [1, 3]                    # 4/7, 3/7
    assert [draw(u, top_p=0.65) for u in (0.5, 0.6)] == [1, 3]                 # 0.4 + 0.3 reach 0.65
    assert [draw(u, top_p=0.75) for u in (0.4, 0.5, 0.7)] == [1, 2, 3]         # 0.2 more: 4/9, 2/9, 3/9
    assert [draw(u, min_p=0.6) for u in (0.5, 0.6)] == [1, 3]
    assert [draw(u, top_k=3, top_p=0.5) for u in (0.5, 0.6)] == [1, 3]         # 0.4 of 0.9 is less than 0.45
    assert [draw(u, temperature=0.5) for u in (0.02, 0.04, 0.5, 0.6, 0.8)] == [0, 1, 1, 2, 3]   # 1, 16, 4, 9 of 30
    _, logp, _ = OO.sample_tokens(x, [0.5], top_k=[2])
    assert abs(logp[0] - np.log(4 / 7)) < 1e-12


def test_largest_arguments(km):  # noqa: F811
    """Workspaces of the largest accepted sizes do not overflow."""
    most = (1 << 31) - 1
    for T, V in ((most, most), (most, 1), (1, most), (0, most)):
        assert 256 <= km.kmp_sample_tokens_workspace_bytes(T, V) < 1 << 62

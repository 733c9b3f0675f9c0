"""The operators on the GPU as a program that keeps its buffers calls them."""
import pytest

from tests.gpu_common import announce, device

pytestmark = pytest.mark.gpu


def test_one_workspace_for_all_batches():
    """The workspace of the largest batch, exactly, serves the smaller ones with
    the results of a workspace of their own; nothing is written behind it."""
    import torch
    from paper_2606_06742_amd import kmpath as km
    gen = torch.Generator(device="cuda")
    gen.manual_seed(3)
    V, top = 70001, 7
    need = km.kmp_token_logprobs_workspace_bytes(1500, V, top)
    kept = torch.full((need + 4096,), 77, dtype=torch.uint8, device=device())
    for T in (1500, 600, 300, 64, 1):
        announce(f"token logprobs {T} x {V} in the workspace of 1500 tokens")
        x = torch.randn(T, V, generator=gen, device=device())
        tok = torch.randint(0, V, (T,), generator=gen, device=device())

        def call(ws):
            lp, H, tl = torch.empty(T, device=device()), torch.empty(T, device=device()), torch.empty(T, top, device=device())
            ti = torch.empty(T, top, dtype=torch.int32, device=device())
            km.kmp_token_logprobs(x, tok, lp, entropy=H, top_id=ti, top_logp=tl, workspace=ws)
            return lp, H, ti, tl

        own = torch.empty(km.kmp_token_logprobs_workspace_bytes(T, V, top), dtype=torch.uint8, device=device())
        assert all(torch.equal(a, b) for a, b in zip(call(kept[:need]), call(own)))
        assert bool((kept[need:] == 77).all())

"""The operators' calls on the host: workspace sizes over the whole range of their
arguments, and what the binding takes for a tensor of the right type and place."""
import os

import pytest


@pytest.fixture(scope="module")
def km():
    from paper_2606_06742_amd import kmpath
    if not os.path.exists(kmpath.LIB_PATH):
        from paper_2606_06742_amd import build
        build.build()
    kmpath.lib()
    return kmpath


def test_workspace_of_no_tokens(km):
    """T = 0 is a valid call, and a size of 0 means bad arguments."""
    for V in (1, 16384, 16385, 128000, 2 ** 31 - 1):
        for top in (0, 1):
            assert km.kmp_token_logprobs_workspace_bytes(0, V, top) > 0, (V, top)

"""The example that runs the operators together with the path: the norm's steps
lower the loss, and the kernel machine tells right answers from wrong ones better
than always guessing the more frequent."""
import importlib.util
import os

import pytest

from tests.gpu_common import announce

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_token_confidence_example():
    spec = importlib.util.spec_from_file_location("token_confidence", os.path.join(ROOT, "examples", "token_confidence.py"))
    ex = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(ex)
    announce("example token_confidence 600 answers, width 250, 3001 tokens")
    r = ex.run(n=600, K=250, V=3001, steps=4)
    assert all(b < a for a, b in zip(r["losses"], r["losses"][1:])), r["losses"]
    assert r["error"] < r["base"], r

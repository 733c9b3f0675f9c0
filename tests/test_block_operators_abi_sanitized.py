"""The host code of the norms around a block, the products with an activation and the
choice of tokens (refusals, workspace sizes, the binding's checks) under
AddressSanitizer and UndefinedBehaviorSanitizer; every call returns before the library
touches a device."""
import os
import shutil
import subprocess
import sys

import pytest

from tests.test_operators_abi_sanitized import ROOT, _library


@pytest.mark.skipif(shutil.which("hipcc") is None and not os.path.exists("/opt/rocm/bin/hipcc"),
                    reason="needs the ROCm compiler")
def test_host_paths_under_asan_and_ubsan():
    from paper_2606_06742_amd import build_sanitized as bs
    env = dict(os.environ)
    env["KMPATH_LIB"] = _library(bs)
    env["LD_PRELOAD"] = bs.runtime()
    env["ASAN_OPTIONS"] = "detect_leaks=0:abort_on_error=1:halt_on_error=1"
    env["UBSAN_OPTIONS"] = "halt_on_error=1:print_stacktrace=1"
    files = [os.path.join(ROOT, "tests", f) for f in ("test_block_norm_abi.py", "test_dense_product_abi.py", "test_sample_abi.py")]
    r = subprocess.run([sys.executable, "-m", "pytest", "-q", "-p", "no:cacheprovider", *files],
                       cwd=ROOT, env=env, capture_output=True, text=True, timeout=600)
    out = r.stdout[-4000:] + r.stderr[-4000:]
    assert r.returncode == 0, out
    assert "passed" in r.stdout and "ERROR: AddressSanitizer" not in out and "runtime error" not in out

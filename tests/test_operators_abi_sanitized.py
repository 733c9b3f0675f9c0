"""The operators' entry points on the host (refusals, workspace sizes up to the
largest accepted arguments, the binding's checks) run against the build with
AddressSanitizer and UndefinedBehaviorSanitizer on its host code. Every call in
those tests returns before the library touches a device."""
import os
import shutil
import subprocess
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def _library(bs):
    """The sanitized library: the one that is there where no source is newer."""
    files = bs.sources() + [os.path.join(d, f) for d in (bs.CSRC, bs.INCLUDE) for f in os.listdir(d)] + [bs.__file__]
    if os.path.exists(bs.LIB) and os.path.getmtime(bs.LIB) > max(os.path.getmtime(f) for f in files):
        return bs.LIB
    return bs.build()


@pytest.mark.skipif(shutil.which("hipcc") is None and not os.path.exists("/opt/rocm/bin/hipcc"),
                    reason="needs the ROCm compiler")
def test_operator_host_paths_under_asan_and_ubsan():
    from paper_2606_06742_amd import build_sanitized as bs
    env = dict(os.environ)
    env["KMPATH_LIB"] = _library(bs)
    env["LD_PRELOAD"] = bs.runtime()
    env["ASAN_OPTIONS"] = "detect_leaks=0:abort_on_error=1:halt_on_error=1"
    env["UBSAN_OPTIONS"] = "halt_on_error=1:print_stacktrace=1"
    r = subprocess.run([sys.executable, "-m", "pytest", "-q", "-p", "no:cacheprovider",
                        os.path.join(ROOT, "tests", "test_operators_abi.py"),
                        os.path.join(ROOT, "tests", "test_operators_calls.py")],
                       cwd=ROOT, env=env, capture_output=True, text=True, timeout=600)
    out = r.stdout[-4000:] + r.stderr[-4000:]
    assert r.returncode == 0, out
    assert "passed" in r.stdout and "ERROR: AddressSanitizer" not in out and "runtime error" not in out

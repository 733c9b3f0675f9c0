"""What the entry points of the norms around a block pass on to their launchers, without
a device: the launchers are replaced by ones that report a gate per row."""
import os
import shutil
import subprocess
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HIPCC = "/opt/rocm/bin/hipcc" if os.path.exists("/opt/rocm/bin/hipcc") else shutil.which("hipcc")

LAUNCHERS = r"""
#include "kmp_operators.h"
namespace kmp {
int block_forward(hipStream_t, const BlockArgs& a) { return a.ldg == 0 ? 100 : 101; }
int block_backward(hipStream_t, const BlockBackArgs& a) { return a.ldg == 0 ? 100 : 101; }
}
"""

CALLS = r"""
import ctypes, sys
ctypes.CDLL(sys.argv[1], mode=ctypes.RTLD_GLOBAL)        # before the library, whose calls then go there
from paper_2606_06742_amd import kmpath as km
L, P = km.lib(), 1 << 20
def forward(gate, ldg):
    return L.kmp_block_norm(None, 2, 2, P, 8, P, 8, 4, 8, 2, None, None, gate, ldg, 1.0, None, None, 1e-5, P + 64, 8, 2, P + 128, 8,
                            None, None)
def backward(gate, ldg):
    return L.kmp_block_norm_backward(None, 2, 2, P, 8, P, 8, P, 8, P, 8, 4, 8, 2, None, None, gate, ldg, 1.0, None, P, P + 64, 8,
                                     P + 128, 8, None, 8, None, None, None, None, None, 0)
for call in (forward, backward):
    print(call.__name__, [call(P, 0), call(P, 8), call(None, 0), call(None, 8), call(None, -1)])
"""


@pytest.mark.skipif(HIPCC is None, reason="needs the ROCm compiler")
def test_no_gate_has_no_rows(tmp_path):
    """A gate that is NULL is one for all rows, whatever its leading dimension."""
    source, library = tmp_path / "launchers.cpp", tmp_path / "liblaunchers.so"
    source.write_text(LAUNCHERS)
    subprocess.run([HIPCC, "--offload-arch=gfx950", "--offload-host-only", "-std=c++17", "-fPIC", "-shared", "-I", os.path.join(ROOT, "include"), "-I",
                    os.path.join(ROOT, "paper_2606_06742_amd", "csrc"), "-x", "hip", str(source), "-o", str(library)],
                   check=True, capture_output=True, timeout=300)
    r = subprocess.run([sys.executable, "-c", CALLS, str(library)], cwd=ROOT, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stderr
    assert r.stdout.split("\n")[:2] == [f"{name} [100, 101, 100, 100, 100]" for name in ("forward", "backward")], r.stdout

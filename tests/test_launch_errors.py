"""A launch that fails is reported by the call that made it: scores of tokens and embedding,
with a stand-in for the runtime's launch (tests/sanitize/launch_errors_driver.cpp; CPU only)."""
import os
import subprocess

import pytest

import paper_2010_10458_amd as tk
from paper_2010_10458_amd import build

HERE = os.path.dirname(os.path.abspath(__file__))


@pytest.mark.skipif(not os.path.exists(build.HIPCC), reason="hipcc not available")
def test_launch_errors_are_reported(tmp_path):
    tk.lib()        # (built, if it was not)
    exe = str(tmp_path / "launch_errors_driver")
    cmd = [build.HIPCC, "--offload-arch=gfx950", "-O1", "-std=c++17", "-rdynamic",
           "-I" + os.path.join(build.ROOT, "include"),
           os.path.join(HERE, "sanitize", "launch_errors_driver.cpp"),
           "-L" + build.LIBDIR, "-ltkef", "-Wl,-rpath," + build.LIBDIR, "-o", exe]
    p = subprocess.run(cmd, capture_output=True, text=True, timeout=600)
    assert p.returncode == 0, p.stderr[-4000:]
    r = subprocess.run([exe], capture_output=True, text=True, timeout=120)
    assert r.returncode == 0 and "0 failed checks" in r.stdout, r.stderr[-2000:]

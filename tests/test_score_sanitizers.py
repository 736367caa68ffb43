"""The host code of the scores of tokens and of the embedding under AddressSanitizer and
UndefinedBehaviorSanitizer (CPU only; the sanitizers are on the host side of the build,
the GPU code is neither instrumented nor launched), driven through the C ABI by
tests/sanitize/score_abi_driver.cpp."""
import os
import subprocess

import pytest

from test_host_sanitizers import HIPCC, ROOT, SAN, _run


@pytest.mark.skipif(not os.path.exists(HIPCC), reason="hipcc not available")
def test_score_abi_under_asan_ubsan(tmp_path):
    exe = str(tmp_path / "score_abi_driver")
    csrc = os.path.join(ROOT, "paper_2010_10458_amd", "csrc")
    cmd = [HIPCC, "--offload-arch=gfx950", "-O1", "-g", "-std=c++17",
           "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
           "-Xarch_host", "-fsanitize=address", "-Xarch_host", "-fsanitize=undefined",
           "-Xarch_host", "-fno-sanitize-recover=all", "-fno-omit-frame-pointer",
           "-I" + os.path.join(ROOT, "include"), "-I" + csrc,
           *[os.path.join(csrc, f) for f in ("tkef_score.hip", "tkef_score_api.cpp",
                                             "tkef_embed.hip", "tkef_embed_api.cpp")],
           os.path.join(SAN, "score_abi_driver.cpp"), "-o", exe]
    p = subprocess.run(cmd, capture_output=True, text=True, timeout=600)
    assert p.returncode == 0, p.stderr[-4000:]
    assert "0 failed checks" in _run(exe, leaks=False)

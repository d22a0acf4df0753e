"""AddressSanitizer + UndefinedBehaviorSanitizer over the host-only parts of include/symb_loss.h (as tests/test_sanitizers.py does for the rest of the library).  GPU code is not instrumented."""
import os
import subprocess

from test_sanitizers import ROOT, SAN, _run


def test_loss_host_code_under_asan_and_ubsan(tmp_path):
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
    exe = str(tmp_path / "loss_san")
    cmd = [hipcc, "-O1", "-g", "-std=c++17", "--offload-arch=gfx950", "-Xarch_device", "-O3", "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
           "-Xarch_host", "-fsanitize=address", "-Xarch_host", "-fsanitize=undefined", "-Xarch_host", "-fno-sanitize-recover=all", "-fno-omit-frame-pointer",
           "-o", exe, os.path.join(SAN, "loss_san.cpp"), os.path.join(ROOT, "paper_2507_03220_amd", "csrc", "symb_loss.hip")]
    r = subprocess.run(cmd, capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-4000:]
    _run(exe)

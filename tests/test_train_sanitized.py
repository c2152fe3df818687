"""The training operators' host code (csrc/train_capi.hip) under AddressSanitizer and UBSan:
tests/host_check/train_host_check.cpp drives every call against stubs of the launchers.
Sanitizers apply to host code only."""

import os
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HIPCC = "/opt/rocm/bin/hipcc"
CLANG = "/opt/rocm/llvm/bin/clang++"


@pytest.mark.skipif(not (os.path.exists(HIPCC) and os.path.exists(CLANG)), reason="ROCm compilers not found")
def test_train_host_paths_under_asan_and_ubsan(tmp_path):
    capi = os.path.join(ROOT, "paper_2107_03356_amd", "csrc", "train_capi.hip")
    drv = os.path.join(ROOT, "tests", "host_check", "train_host_check.cpp")
    san = ["-fsanitize=address", "-fsanitize=undefined", "-fno-sanitize-recover=undefined"]
    host_san = [a for f in san for a in ("-Xarch_host", f)]
    common = ["-std=c++17", "-O1", "-g", "-fno-omit-frame-pointer"]
    cmds = [
        [HIPCC, *common, "--offload-arch=gfx950", "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
         *host_san, "-c", capi, "-o", str(tmp_path / "capi.o")],
        [CLANG, *common, *san, "-I/opt/rocm/include", "-D__HIP_PLATFORM_AMD__", "-c", drv, "-o", str(tmp_path / "check.o")],
        [CLANG, *san, str(tmp_path / "capi.o"), str(tmp_path / "check.o"), "-o", str(tmp_path / "check")],
    ]
    for c in cmds:
        r = subprocess.run(c, capture_output=True, text=True)
        assert r.returncode == 0, (" ".join(c), r.stderr[-4000:])
    r = subprocess.run([str(tmp_path / "check")], capture_output=True, text=True, timeout=300)
    out = r.stdout + r.stderr
    assert r.returncode == 0 and "host check ok" in r.stdout, out[-6000:]
    assert "AddressSanitizer" not in out and "runtime error" not in out, out[-6000:]

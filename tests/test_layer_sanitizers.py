"""The host side of the entry points of include/gt_layer.h under AddressSanitizer
(CPU only): tests/sanitize/layer_driver.cpp and the library's host code, over the
stand-in runtime tests/sanitize/hip_stub.cpp."""
import os
import re
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
SAN = os.path.join(ROOT, "tests", "sanitize")
ROCM = os.environ.get("ROCM_PATH", "/opt/rocm")


def test_layer_host_side_under_asan(tmp_path):
    llvm, hipcc = os.path.join(ROCM, "lib", "llvm", "bin"), os.path.join(ROCM, "bin", "hipcc")
    if not os.path.exists(hipcc) or not os.path.exists(os.path.join(llvm, "clang++")):
        pytest.skip("hipcc not available")
    inc = ["-D__HIP_PLATFORM_AMD__", "-isystem", os.path.join(ROCM, "include"), "-I", os.path.join(ROOT, "include")]

    def run(cmd):
        r = subprocess.run(cmd, capture_output=True, text=True, timeout=900, cwd=tmp_path)
        assert r.returncode == 0, (r.stdout + r.stderr)[-4000:]
        return r.stdout

    run([hipcc, "--offload-arch=gfx950", "--offload-host-only", "-O1", "-g", "-std=c++17", "-Xarch_host", "-fsanitize=address",
         "-I", os.path.join(ROOT, "include"), "-c", os.path.join(ROOT, "paper_2605_31500_amd", "csrc", "gt_attn.hip"), "-o", "lib.o"])
    for src in ("hip_stub.cpp", "layer_driver.cpp"):
        run([os.path.join(llvm, "clang++"), "-std=c++17", "-O1", "-g", "-fno-omit-frame-pointer", "-fsanitize=address"] + inc
            + ["-c", os.path.join(SAN, src), "-o", src + ".o"])
    image = [l.split()[-1] for l in run(["nm", "lib.o"]).splitlines() if "__hip_fatbin_" in l and " U " in l and "wrapper" not in l]
    run([os.path.join(llvm, "clang++"), "-fsanitize=address", "lib.o", "hip_stub.cpp.o", "layer_driver.cpp.o", "-lm", "-lpthread",
         "-o", "prog"] + ["-Wl,--defsym=%s=0" % s for s in image])
    r = subprocess.run([str(tmp_path / "prog")], capture_output=True, text=True, timeout=300,
                       env=dict(os.environ, ASAN_OPTIONS="detect_leaks=1"))
    out = r.stdout + r.stderr
    assert r.returncode == 0 and "0 failure(s)" in out, out[-4000:]
    assert "AddressSanitizer" not in out and re.search(r"hip stub: [1-9]\d* launches, 0 allocations left", out), out[-4000:]

"""The host code of the operators around the layer under AddressSanitizer (no
GPU needed), with a stand-in for the HIP runtime that launches nothing
(tests/ops_host_driver.c): calls over a grid of sizes, among them the largest,
and every launch they make within the device's limits."""
import os
import re
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HIPCC = "/opt/rocm/bin/hipcc"


@pytest.mark.skipif(not os.path.exists(HIPCC), reason="hipcc not installed")
def test_ops_host_paths_under_asan(tmp_path):
    src = os.path.join(ROOT, "paper_2608_10392_amd", "csrc", "ops.hip")
    obj, exe = tmp_path / "ops_host.o", tmp_path / "ops_host"
    asan = ["-Xarch_host", "-fsanitize=address", "-Xarch_host", "-fno-omit-frame-pointer"]
    subprocess.run([HIPCC, "--offload-arch=gfx950", "--offload-host-only", "-std=c++17", "-O1", "-g", *asan, "-c", src,
                    "-o", str(obj)], check=True, capture_output=True)
    # the device code's place in the object stays empty
    names = re.findall(r"U (__hip_fatbin\w*)", subprocess.run(["nm", "-u", str(obj)], capture_output=True, text=True).stdout)
    stand_in = tmp_path / "fatbin.c"
    stand_in.write_text("".join(f"const char {n}[64];\n" for n in names))
    drv = os.path.join(ROOT, "tests", "ops_host_driver.c")
    subprocess.run([shutil.which("clang") or os.path.join(os.path.dirname(HIPCC), "..", "llvm", "bin", "clang"), "-O1",
                    "-g", "-fsanitize=address", "-I", os.path.join(ROOT, "include"), drv, str(stand_in), str(obj), "-lstdc++",
                    "-lm", "-o", str(exe)], check=True, capture_output=True, text=True)
    env = dict(os.environ, ASAN_OPTIONS="detect_leaks=1:abort_on_error=0:exitcode=23")
    r = subprocess.run([str(exe)], capture_output=True, text=True, env=env, timeout=120)
    assert r.returncode == 0, r.stdout[-4000:] + r.stderr[-4000:]
    assert "ops host paths ok" in r.stdout, r.stdout

"""Refused calls of the operators around the layer make no HIP call (no GPU
needed): the library's host code against a stand-in for the HIP runtime
(tests/ops_refusals_driver.c)."""
import os
import re
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HIPCC = "/opt/rocm/bin/hipcc"
CLANG = "/opt/rocm/llvm/bin/clang"


@pytest.mark.skipif(not os.path.exists(HIPCC), reason="hipcc not installed")
def test_refused_calls_make_no_hip_call(tmp_path):
    src = os.path.join(ROOT, "paper_2608_10392_amd", "csrc", "ops.hip")
    obj, exe = tmp_path / "ops_host.o", tmp_path / "refusals"
    subprocess.run([HIPCC, "--offload-arch=gfx950", "--offload-host-only", "-std=c++17", "-O1", "-c", src, "-o", str(obj)],
                   check=True, capture_output=True)
    # the device code's place in the object stays empty
    names = re.findall(r"U (__hip_fatbin\w*)", subprocess.run(["nm", "-u", str(obj)], capture_output=True, text=True).stdout)
    stand_in = tmp_path / "fatbin.c"
    stand_in.write_text("".join(f"const char {n}[64];\n" for n in names))
    subprocess.run([CLANG, "-O1", "-I", os.path.join(ROOT, "include"), os.path.join(ROOT, "tests", "ops_refusals_driver.c"),
                    str(stand_in), str(obj), "-lstdc++", "-lm", "-o", str(exe)], check=True, capture_output=True, text=True)
    r = subprocess.run([str(exe)], capture_output=True, text=True, timeout=60)
    assert r.returncode == 0, r.stdout[-4000:] + r.stderr[-4000:]
    assert "ops refusals ok" in r.stdout, r.stdout

"""Builds libunifmoe.so, the HIP library for gfx950, in place.

    python -m paper_2608_10392_amd.build
"""
import os
import shutil
import subprocess
import sys

HERE = os.path.dirname(os.path.abspath(__file__))
SRCS = [os.path.join(HERE, "csrc", name) for name in ("unif_moe.hip", "ops.hip")]
LIB = os.path.join(HERE, "libunifmoe.so")

# Packed fp32 VALU instructions are switched off for all device code. The
# atomic optimizer is off: it turns a one-lane atomic with return (the GEMM
# tile queues) into a wave-wide one whose result is broadcast at once, which
# drains every copy in flight.
HIPCC_FLAGS = ["--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC",
               "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
               "-mllvm", "-amdgpu-atomic-optimizer-strategy=None"]


def hipcc():
    path = os.environ.get("HIPCC") or shutil.which("hipcc") or "/opt/rocm/bin/hipcc"
    if not os.path.exists(path):
        raise RuntimeError("hipcc not found; set HIPCC or install ROCm")
    return path


def build(verbose=False):
    """Compiles the sources side by side, then links them into the library."""
    tmp = LIB + ".tmp"
    objs = [LIB + "." + os.path.basename(src) + ".o" for src in SRCS]
    runs = [subprocess.Popen([hipcc()] + HIPCC_FLAGS + ["-c", "-o", obj, src], stdout=subprocess.PIPE,
                             stderr=subprocess.STDOUT, text=True) for src, obj in zip(SRCS, objs)]
    outs = [run.communicate()[0] for run in runs]
    if all(run.returncode == 0 for run in runs):
        link = subprocess.run([hipcc(), "--offload-arch=gfx950", "-fPIC", "-shared", "-o", tmp] + objs,
                              capture_output=True, text=True)
        runs.append(link)
        outs.append(link.stdout + link.stderr)
    for obj in objs:
        if os.path.exists(obj):
            os.remove(obj)
    msgs = [l for l in "".join(outs).splitlines()
            if "packed-fp32-ops' is not a recognized feature" not in l]
    if any(run.returncode != 0 for run in runs):
        raise RuntimeError("hipcc failed:\n" + "\n".join(msgs))
    if verbose and msgs:
        print("\n".join(msgs), file=sys.stderr)
    os.replace(tmp, LIB)
    return LIB


if __name__ == "__main__":
    print(build(verbose=True))

"""Compile the HIP planner for gfx950 into paper_2309_08125_amd/lib/liboob_plan.so."""
from __future__ import annotations

import glob
import os
import subprocess

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
SRC_DIR = os.path.join(HERE, "csrc")
LIB_DIR = os.path.join(HERE, "lib")
LIB = os.path.join(LIB_DIR, "liboob_plan.so")
# The planner's kernels form no NaN (its infinities never meet).  A layer's operators get whatever a model holds.
NO_NANS = ["-fno-honor-nans"]


def sources():
    return sorted(glob.glob(os.path.join(SRC_DIR, "*.hip")))


def build(verbose: bool = False) -> str:
    """Every source on its own (side by side), then one library."""
    os.makedirs(LIB_DIR, exist_ok=True)
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
    flags = ["--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC",
             "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops", "-Wno-unused-command-line-argument",
             "-I", os.path.join(ROOT, "include"), "-I", os.path.join(HERE, "include"), "-I", SRC_DIR]
    running = []
    for src in sources():
        name = os.path.basename(src)[:-len(".hip")]
        obj = os.path.join(LIB_DIR, name + ".o")
        cmd = [hipcc] + flags + ([] if name.startswith("oob_layer_") else NO_NANS) + ["-c", "-o", obj, src]
        if verbose:
            print(" ".join(cmd))
        running.append((cmd, obj, subprocess.Popen(cmd, stdout=subprocess.PIPE, stderr=subprocess.PIPE, text=True)))
    failed = []
    for cmd, obj, p in running:
        err = p.communicate()[1]
        if p.returncode != 0:
            failed.append(err)
        # the host pass warns that it does not know the packed-fp32 feature: harmless
        elif verbose and (err := "\n".join(line for line in err.splitlines() if "packed-fp32-ops" not in line)).strip():
            print(err)
    if not failed:
        cmd = [hipcc, "--offload-arch=gfx950", "-shared", "-fPIC", "-o", LIB] + [obj for _, obj, _ in running]
        if verbose:
            print(" ".join(cmd))
        res = subprocess.run(cmd, capture_output=True, text=True)
        if res.returncode != 0:
            failed.append(res.stderr)
    for _, obj, _ in running:
        if os.path.exists(obj):
            os.remove(obj)
    if failed:
        raise RuntimeError("hipcc failed:\n" + "\n".join(failed))
    return LIB


def ensure_built() -> str:
    """Builds only if no library is there (tests, smoke and bench call this; a changed source
    needs an explicit build)."""
    return LIB if os.path.exists(LIB) else build()


if __name__ == "__main__":
    print(build(verbose=True))

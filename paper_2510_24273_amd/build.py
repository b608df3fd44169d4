"""Build libsals.so (HIP kernels + C ABI) for gfx950 with hipcc, in-tree."""
from __future__ import annotations

import os
import subprocess
import sys
import tempfile

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libsals.so")

HIPCC_FLAGS = [
    "-O3", "-std=c++17", "--offload-arch=gfx950", "-fPIC", "-shared",
    # keep hipcc from forming packed-fp32 instructions
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    # the first kernel arguments arrive in scalar registers with the wave instead of through scalar loads at its
    # start (as many as the hardware's user registers allow; measured: 1.2 us of the 38 us step at B = 1)
    "-mllvm", "-amdgpu-kernarg-preload-count=16",
    "-Wall", "-Wno-unused-function",
]


def sources():
    return [os.path.join(CSRC, f) for f in sorted(os.listdir(CSRC)) if f.endswith(".hip")]


def headers():
    inc = os.path.join(os.path.dirname(HERE), "include")
    return [os.path.join(CSRC, f) for f in os.listdir(CSRC) if f.endswith(".hpp")] + \
           [os.path.join(inc, f) for f in os.listdir(inc)]


def is_stale() -> bool:
    if not os.path.exists(LIB):
        return True
    t = os.path.getmtime(LIB)
    return any(os.path.getmtime(f) > t for f in sources() + headers())


def build(force: bool = True, verbose: bool = False) -> str:
    """Compile every HIP source into libsals.so; returns its path."""
    if not force and not is_stale():
        return LIB
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
    added = os.environ.get("SALS_EXTRA_FLAGS", "").split()   # (for the link as well: sanitizers, libraries)
    flags = HIPCC_FLAGS + added
    with tempfile.TemporaryDirectory() as tmp:   # the sources side by side, then one link in the order of their names
        jobs, objs = [], []
        for src in sources():
            objs.append(os.path.join(tmp, os.path.basename(src) + ".o"))
            cmd = [hipcc] + [f for f in flags if f != "-shared"] + ["-c", src, "-o", objs[-1]]
            if verbose:
                print(" ".join(cmd), flush=True)
            jobs.append((cmd, subprocess.Popen(cmd)))
        failed = [(cmd, p.returncode) for cmd, p in jobs if p.wait() != 0]
        if failed:
            raise subprocess.CalledProcessError(failed[0][1], failed[0][0])
        subprocess.run([hipcc, "-shared", "-fPIC", "--offload-arch=gfx950", "-o", LIB] + objs + added, check=True)
    return LIB


if __name__ == "__main__":
    print(build(force=True, verbose=True))
    sys.exit(0)

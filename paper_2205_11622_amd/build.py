"""Builds libsparselnr.so (HIP, gfx950) in place.

    python -m paper_2205_11622_amd.build

Every call recompiles.  Packed-FP32 instruction selection is disabled for
all device code (-packed-fp32-ops).
"""
from __future__ import annotations

import os
import shutil
import subprocess
import sys
import tempfile

PKG = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(PKG)
CSRC = os.path.join(PKG, "csrc")    # the sparse products
PAGED = os.path.join(PKG, "paged")  # attention over a paged cache
INCLUDE = os.path.join(ROOT, "include")
LIB = os.path.join(PKG, "libsparselnr.so")
ARCH = "gfx950"


def hipcc() -> str:
    for cand in (os.environ.get("HIPCC"), shutil.which("hipcc"), "/opt/rocm/bin/hipcc"):
        if cand and os.path.exists(cand):
            return cand
    raise RuntimeError("hipcc not found")


def flags() -> list:
    return ["--offload-arch=" + ARCH, "-O3", "-std=c++17", "-fPIC",
            "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
            "-fvisibility=hidden", "-Wall", "-Wno-unused-result", "-I", INCLUDE, "-I", CSRC]


def sources() -> list:
    """paged/library.hip takes csrc/sparselnr.hip in."""
    return sorted(os.path.join(PAGED, f) for f in os.listdir(PAGED) if f.endswith(".hip"))


def build(verbose: bool = False) -> str:
    tmp = LIB + ".tmp%d" % os.getpid()
    with tempfile.TemporaryDirectory() as work:
        objects, running = [], []
        for src in sources():  # at once: the largest takes as long as all others
            objects.append(os.path.join(work, os.path.basename(src) + ".o"))
            cmd = [hipcc(), *flags(), "-c", src, "-o", objects[-1]]
            if verbose:
                print(" ".join(cmd), flush=True)
            running.append((cmd, subprocess.Popen(cmd)))
        for cmd, p in running:
            p.wait()
        for cmd, p in running:
            if p.returncode != 0:
                raise subprocess.CalledProcessError(p.returncode, cmd)
        subprocess.check_call([hipcc(), "--offload-arch=" + ARCH, "-shared", *objects, "-o", tmp])
    os.replace(tmp, LIB)
    return LIB


if __name__ == "__main__":
    print(build(verbose=True))
    sys.exit(0)

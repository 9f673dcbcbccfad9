"""Compile the HIP library for gfx950 into paper_2312_17238_amd/libmoe_offload.so."""
from __future__ import annotations

import glob
import os
import subprocess
import tempfile

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libmoe_offload.so")
SOURCES = [os.path.join(CSRC, "moe_offload.hip"), os.path.join(CSRC, "kv.hip")]
HEADERS = glob.glob(os.path.join(CSRC, "*.h")) + glob.glob(os.path.join(os.path.dirname(HERE), "include", "*.h"))

FLAGS = [
    "-O3", "-std=c++17", "-fPIC", "--offload-arch=gfx950",
    "-munsafe-fp-atomics", "-pthread",
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    "-Wall", "-Wno-unused-function",
]


def stale() -> bool:
    if not os.path.exists(LIB):
        return True
    t = os.path.getmtime(LIB)
    return any(os.path.getmtime(p) > t for p in SOURCES + HEADERS)


def build(force: bool = True, extra=()) -> str:
    """Compiles every time unless force=False and the library is newer than its sources."""
    if force or stale():
        hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
        with tempfile.TemporaryDirectory() as tmp:     # the sources at the same time, each into an object of its own
            objects = [os.path.join(tmp, os.path.basename(s) + ".o") for s in SOURCES]
            jobs = [subprocess.Popen([hipcc, *FLAGS, *extra, "-c", "-o", o, s]) for s, o in zip(SOURCES, objects)]
            codes = [j.wait() for j in jobs]
            if any(codes):
                raise RuntimeError(f"hipcc failed on {[os.path.basename(s) for s, c in zip(SOURCES, codes) if c]}")
            subprocess.check_call([hipcc, "-shared", "-fPIC", "--offload-arch=gfx950", "-pthread", "-o", LIB, *objects])
    return LIB


if __name__ == "__main__":
    import sys
    print(build(True, sys.argv[1:]))

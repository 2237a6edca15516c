"""Builds libhufflm.so (host codec + gfx950 kernels) in place with hipcc."""
from __future__ import annotations

import os
import subprocess
import sys
import tempfile
from concurrent.futures import ThreadPoolExecutor

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libhufflm.so")
SOURCES = ["kernels.hip", "norm.hip", "attention.hip", "evict.hip", "host_codec.cpp"]
HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")

FLAGS = [
    "-O3", "-std=c++17", "-fPIC", "--offload-arch=gfx950",
    # keep packed-fp32 instructions out of the device code
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    "-munsafe-fp-atomics",
    "-Wall", "-Wno-unused-result",
]
# the prefill product of many tokens multiplies the decoded weights with hipBLASLt
LINK = ["-shared", "-fPIC", "--offload-arch=gfx950", "-lhipblaslt"]


def build(verbose: bool = False) -> str:
    """Compiles each source on its own, all at once, and links them."""
    def run(cmd):
        if verbose:
            print(" ".join(cmd), flush=True)
        r = subprocess.run(cmd, capture_output=True, text=True)
        noise = "is not a recognized feature for this target"
        err = "\n".join(l for l in (r.stderr or "").splitlines() if noise not in l)
        if r.returncode != 0:
            raise RuntimeError(f"hipcc failed ({r.returncode}):\n{err}")
        if verbose and err.strip():
            print(err, file=sys.stderr)

    tmp = LIB + ".tmp"
    with tempfile.TemporaryDirectory() as folder, ThreadPoolExecutor(len(SOURCES)) as pool:
        objects = [os.path.join(folder, s + ".o") for s in SOURCES]
        include = ["-I", os.path.join(ROOT, "include"), "-I", CSRC]
        list(pool.map(run, [[HIPCC, *FLAGS, *include, "-c", os.path.join(CSRC, s), "-o", o]
                            for s, o in zip(SOURCES, objects)]))
        run([HIPCC, *LINK, *objects, "-o", tmp])
    os.replace(tmp, LIB)
    return LIB


if __name__ == "__main__":
    print(build(verbose=True))

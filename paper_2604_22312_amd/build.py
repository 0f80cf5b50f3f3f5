"""Build the gfx950 shared library ``libgvr_topk.so`` in-tree with hipcc."""
from __future__ import annotations

import os
import subprocess
import sys
import tempfile
from concurrent.futures import ThreadPoolExecutor

PKG = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(PKG)
SOURCES = [os.path.join(PKG, "csrc", f) for f in ("gvr_topk.hip", "rope_prior.hip", "indexer.hip", "read_floor.hip",
                                                 "rotary.hip", "kv4_cache.hip", "kv4_attention.hip",
                                                 "pages.hip", "fp8_quantize.hip", "fp8_matmul.hip")]
INCLUDE = os.path.join(ROOT, "include")
LIB = os.path.join(PKG, "libgvr_topk.so")
ARCH = "gfx950"

HIPCC_FLAGS = [
    "--offload-arch=" + ARCH, "-O3", "-std=c++17", "-fPIC",
    # packed fp32 VALU forms are kept out of every build of this library
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    # the first 14 dwords of scalar kernel arguments arrive in SGPRs
    "-mllvm", "-amdgpu-kernarg-preload-count=14",
    "-Wall", "-Wno-unused-command-line-argument",
]


def hipcc() -> str:
    for c in ("/opt/rocm/bin/hipcc", "hipcc"):
        if os.path.exists(c) or c == "hipcc":
            return c
    raise RuntimeError("hipcc not found")


def build(verbose: bool = False) -> str:
    """Compile the ``csrc/*.hip`` sources (side by side) into ``libgvr_topk.so`` (always rebuilds)."""
    tmp = LIB + ".tmp%d" % os.getpid()

    def run(cmd):
        if verbose:
            print(" ".join(cmd), flush=True)
        r = subprocess.run(cmd, capture_output=True, text=True)
        if r.returncode != 0:
            sys.stderr.write(r.stdout + r.stderr)
            raise RuntimeError("hipcc failed building %s" % LIB)

    with tempfile.TemporaryDirectory() as objs:
        out = [os.path.join(objs, os.path.basename(f) + ".o") for f in SOURCES]
        with ThreadPoolExecutor(min(len(SOURCES), os.cpu_count() or 1, 8)) as pool:
            list(pool.map(run, [[hipcc()] + HIPCC_FLAGS + ["-I" + INCLUDE, "-c", f, "-o", o]
                                for f, o in zip(SOURCES, out)]))
        run([hipcc(), "--offload-arch=" + ARCH, "-shared", "-o", tmp] + out)
    os.replace(tmp, LIB)
    return LIB


if __name__ == "__main__":
    print(build(verbose=True))

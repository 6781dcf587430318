"""Builds libtt_emb.so (HIP, gfx950 only) in-tree with hipcc."""
from __future__ import annotations

import glob
import os
import subprocess
import tempfile
from concurrent.futures import ThreadPoolExecutor

PKG = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(PKG)
LIB = os.path.join(PKG, "libtt_emb.so")

HIPCC_FLAGS = [
    "-O3", "-std=c++17", "--offload-arch=gfx950", "-fPIC", "-shared", "-munsafe-fp-atomics",
    # keep the compiler from forming packed-fp32 instructions (some of their forms have given wrong
    # results on this hardware); hipcc's host pass warns that it does not know the feature, harmlessly
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    "-Wall", "-Wno-unused-function",
]


def sources():
    return sorted(glob.glob(os.path.join(PKG, "csrc", "*.hip")))


def build(verbose: bool = False) -> str:
    """Compile every HIP source (side by side) and link libtt_emb.so.  Always compiles."""
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
    include = ["-I", os.path.join(ROOT, "include"), "-I", os.path.join(PKG, "csrc")]

    def run(cmd):
        if verbose:
            print(" ".join(cmd), flush=True)
        res = subprocess.run(cmd, capture_output=True, text=True)
        if res.returncode != 0:
            raise RuntimeError("hipcc failed:\n" + res.stdout + res.stderr)
        if verbose and res.stderr.strip():
            print(res.stderr)

    with tempfile.TemporaryDirectory() as tmp:
        jobs = [(src, os.path.join(tmp, os.path.basename(src) + ".o")) for src in sources()]
        compile_flags = [f for f in HIPCC_FLAGS if f != "-shared"]
        workers = int(os.environ.get("MAX_JOBS") or 0) or min(8, os.cpu_count() or 1)
        with ThreadPoolExecutor(max_workers=workers) as pool:
            list(pool.map(lambda job: run([hipcc] + compile_flags + include + ["-c", job[0], "-o", job[1]]), jobs))
        run([hipcc, "-shared", "-fPIC", "--offload-arch=gfx950", "-o", LIB] + [obj for _, obj in jobs])
    return LIB


if __name__ == "__main__":
    print(build(verbose=True))

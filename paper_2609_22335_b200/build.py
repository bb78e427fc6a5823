"""In-tree build of the CUDA library (sm_100a) with nvcc; no JIT cache involved."""
from __future__ import annotations

import os
import subprocess
import sys
import tempfile

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libvla_b200.so")
SOURCES = ["vla_api.cu", "ops_sequences.cu", "program.cc"]
HEADERS = []


def _stale() -> bool:
    if not os.path.exists(LIB):
        return True
    t = os.path.getmtime(LIB)
    for f in os.listdir(CSRC):
        if os.path.getmtime(os.path.join(CSRC, f)) > t:
            return True
    return os.path.getmtime(os.path.join(HERE, "..", "include", "vla.h")) > t


def build(force: bool = False, verbose: bool = False) -> str:
    if not force and not _stale():
        return LIB
    nvcc = os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")
    flags = ["-std=c++17", "-O3", "-lineinfo", "-gencode", "arch=compute_100a,code=sm_100a", "-Xcompiler", "-fPIC", "-DVLA_EXPORTS",
             # no implicit multiply-add contraction: the same tile body is compiled into several kernels (the
             # persistent one, the per-node ones, the single-op ones) and must round identically in all of them;
             # the fused multiply-adds the bodies want are written as fmaf()
             "-fmad=false"]
    if verbose:
        flags += ["-Xptxas", "-v"]
    with tempfile.TemporaryDirectory() as objects:                  # (an object for each source, side by side)
        out = [os.path.join(objects, s + ".o") for s in SOURCES]
        steps = [subprocess.Popen([nvcc, *flags, "-x", "cu", "-c", "-o", o, os.path.join(CSRC, s)], stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
                 for s, o in zip(SOURCES, out)]
        said = [p.communicate()[0] for p in steps]
        if all(p.returncode == 0 for p in steps):
            link = subprocess.run([nvcc, "-shared", "-gencode", "arch=compute_100a,code=sm_100a", "-o", LIB, *out, "-lcudart"], capture_output=True, text=True)
            said.append(link.stdout + link.stderr)
            steps.append(link)
        if any(p.returncode != 0 for p in steps):
            sys.stderr.write("".join(said))
            raise RuntimeError("nvcc failed building libvla_b200.so")
    if verbose:
        sys.stderr.write("".join(said))
    return LIB


if __name__ == "__main__":
    print(build(force=True, verbose="-v" in sys.argv))

"""Build liblipz.so (HIP, gfx950) in place.

    python -m paper_1811_12843_amd.build
"""
import glob
import os
import shutil
import subprocess
import sys
import tempfile
from concurrent.futures import ThreadPoolExecutor

PKG = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(PKG)
LIB = os.path.join(PKG, "liblipz.so")

HIPCC_FLAGS = [
    "-O3", "-std=c++17", "-fPIC", "-shared",
    "--offload-arch=gfx950",
    # keep packed-fp32 instructions out of the generated code
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    # the first 14 words of kernel arguments arrive preloaded in scalar
    # registers (the GEMM kernels' descriptor pointer, tile groups and step)
    "-mllvm", "-amdgpu-kernarg-preload-count=14",
    "-Wno-unused-command-line-argument",
]


def hipcc():
    h = shutil.which("hipcc") or "/opt/rocm/bin/hipcc"
    if not os.path.exists(h):
        raise RuntimeError("hipcc not found")
    return h


def sources():
    return sorted(glob.glob(os.path.join(PKG, "csrc", "*.hip")))


def build(verbose=False, out=None, defines=()):
    """Compile every HIP source into paper_1811_12843_amd/liblipz.so (or `out`),
    with optional -D definitions.  The sources are compiled side by side, each
    into an object file of its own, and linked."""
    lib = out or LIB
    tmp = lib + ".tmp"
    flags = [*HIPCC_FLAGS, *["-D" + d for d in defines], "-I", os.path.join(ROOT, "include"),
             "-I", os.path.join(PKG, "csrc")]
    msgs = []

    def run(cmd):
        r = subprocess.run(cmd, capture_output=True, text=True)
        text = "\n".join(l for l in (r.stdout + r.stderr).splitlines()
                         if "packed-fp32-ops" not in l and "is not a recognized feature" not in l)
        if r.returncode != 0:
            raise RuntimeError("hipcc failed:\n" + text)
        msgs.append(text)

    with tempfile.TemporaryDirectory() as d:
        jobs = [(src, os.path.join(d, os.path.basename(src) + ".o")) for src in sources()]
        compiles = [[hipcc(), *[f for f in flags if f != "-shared"], "-c", src, "-o", obj] for src, obj in jobs]
        if verbose:
            print(*(" ".join(c) for c in compiles), sep="\n", flush=True)
        with ThreadPoolExecutor(min(8, os.cpu_count() or 1)) as pool:
            list(pool.map(run, compiles))
        run([hipcc(), *HIPCC_FLAGS, *[obj for _, obj in jobs], "-o", tmp])
    if verbose and any(m.strip() for m in msgs):
        print("\n".join(m for m in msgs if m.strip()))
    os.replace(tmp, lib)
    return lib


if __name__ == "__main__":
    print(build(verbose="-v" in sys.argv))

"""Compile libisoloco.so (host planner + gfx950 HIP kernels) in place.

Usage: ``python paper_2607_03011_amd/build.py`` or ``__graft_entry__.build()``.
The library is always rebuilt; tests, the smoke check and the benchmark only
load what is already built.
"""
import os
import subprocess
import sys
import tempfile
from concurrent.futures import ThreadPoolExecutor

PKG = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(PKG)
LIB = os.path.join(PKG, "libisoloco.so")
SOURCES = [os.path.join(PKG, "csrc", f) for f in (
    "isoloco_host.cpp", "isoloco_kernels.hip", "isoloco_products.hip",
    "isoloco_clip.hip", "isoloco_embedding.hip", "isoloco_logprob.hip", "isoloco_ffn.hip", "isoloco_ffn_tiles.hip",
    "isoloco_route.hip", "isoloco_experts.hip", "isoloco_experts_tiles.hip",
    "isoloco_combine.hip", "isoloco_distill.hip")]

HIPCC_FLAGS = [
    "-O3", "-std=c++17", "-fPIC", "-shared", "--offload-arch=gfx950",
    # no packed fp32 instructions in device code
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    "-Wall", "-Wno-unused-result",
]


def _run(cmd, verbose):
    if verbose:
        print(" ".join(cmd), flush=True)
    res = subprocess.run(cmd, capture_output=True, text=True)
    out = "\n".join(l for l in (res.stdout + res.stderr).splitlines()
                    if "packed-fp32-ops" not in l and l.strip())
    if res.returncode != 0:
        raise RuntimeError("hipcc failed (%d):\n%s" % (res.returncode, out))
    if verbose and out:
        print(out, flush=True)


def build(verbose=False):
    """Every source compiled to an object of its own, side by side, then linked."""
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
    tmp = LIB + ".tmp"
    with tempfile.TemporaryDirectory(prefix="isoloco_build_") as d:
        objects = [os.path.join(d, os.path.basename(src) + ".o") for src in SOURCES]
        compile_flags = [f for f in HIPCC_FLAGS if f != "-shared"]
        includes = ["-I", os.path.join(ROOT, "include"), "-I", os.path.join(PKG, "csrc")]
        with ThreadPoolExecutor(max_workers=4) as pool:
            for job in [pool.submit(_run, [hipcc, *compile_flags, *includes, "-c", src, "-o", obj], verbose)
                        for src, obj in zip(SOURCES, objects)]:
                job.result()
        _run([hipcc, "-shared", "-fPIC", "--offload-arch=gfx950", *objects, "-o", tmp], verbose)
    os.replace(tmp, LIB)
    return LIB


if __name__ == "__main__":
    print(build(verbose="-v" in sys.argv))

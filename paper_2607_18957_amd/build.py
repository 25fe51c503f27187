"""Build libii.so (host planner + runtime + gfx950 kernels) with hipcc.

Usage: ``python -m paper_2607_18957_amd.build`` or ``build()`` from Python.
The library is written next to this file so it travels with the source tree.
"""
from __future__ import annotations

import os
import shutil
import subprocess
import sys
import tempfile
from concurrent.futures import ThreadPoolExecutor

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(HERE, "csrc")
INCLUDE = os.path.join(ROOT, "include")
LIB = os.path.join(HERE, "libii.so")
SOURCES = ["plan.cpp", "scatter.hip", "runtime.hip", "ops.cpp", "linear.hip", "cache.hip",
           "attend.hip", "attend_many.hip", "norm.hip", "rotate.hip", "logprobs.hip",
           "adapt.hip"]
ARCH = os.environ.get("II_OFFLOAD_ARCH", "gfx950")

FLAGS = [
    f"--offload-arch={ARCH}", "-O3", "-std=c++17", "-fPIC", "-Wall",
    # packed fp32 instructions are disabled for all device code built here
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
]
LINK = [f"--offload-arch={ARCH}", "-fPIC", "-shared", "-Wl,-soname,libii.so"]


def hipcc() -> str:
    for c in (os.environ.get("HIPCC"), "/opt/rocm/bin/hipcc", shutil.which("hipcc")):
        if c and os.path.exists(c):
            return c
    raise RuntimeError("hipcc not found (ROCm is required to build libii.so)")


def _run(cmd, verbose: bool) -> None:
    if verbose:
        print(" ".join(cmd), flush=True)
    r = subprocess.run(cmd, capture_output=True, text=True)
    noise = "packed-fp32-ops"  # the host pass does not know the feature; harmless
    msgs = "\n".join(l for l in (r.stdout + r.stderr).splitlines() if noise not in l)
    if r.returncode != 0:
        raise RuntimeError(f"hipcc failed ({r.returncode}):\n{msgs}")
    if verbose and msgs.strip():
        print(msgs)


def build(verbose: bool = False) -> str:
    """Compile every source (always recompiles; some at once) and link libii.so."""
    tmp = LIB + f".tmp{os.getpid()}"
    cc = hipcc()
    with tempfile.TemporaryDirectory() as objects:
        jobs = [(os.path.join(CSRC, s), os.path.join(objects, s + ".o")) for s in SOURCES]
        with ThreadPoolExecutor(max_workers=min(8, os.cpu_count() or 1)) as pool:
            for f in [pool.submit(_run, [cc, *FLAGS, "-I", INCLUDE, "-I", CSRC, "-c", "-o", o, s], verbose)
                      for s, o in jobs]:
                f.result()
        _run([cc, *LINK, "-o", tmp, *[o for _, o in jobs]], verbose)
    os.replace(tmp, LIB)
    return LIB


if __name__ == "__main__":
    print(build(verbose="-v" in sys.argv))

"""Build libezsp.so (HIP for gfx950) in the package directory.

Every source is compiled with hipcc and linked into one shared library that
exports the C ABI of ``include/ezsp.h``.  Floating-point contraction is off
(gains and distances must be single IEEE roundings, as the partition's
decisions are compared bit for bit) and packed-fp32 instructions are not
generated.
"""
from __future__ import annotations

import os
import shutil
import subprocess
import sys

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libezsp.so")
BUILD = os.path.join(HERE, "_build")
SOURCES = ["ezsp_prims.hip", "ezsp_knn.hip", "ezsp_merge.hip",
           "ezsp_stats.hip", "ezsp_grid.hip", "ezsp_loss.hip",
           "ezsp_purity.hip", "ezsp_mlp.hip", "ezsp_noalloc.hip",
           "ezsp_norm.hip", "ezsp_linear.hip", "ezsp_gated.hip",
           "ezsp_api.hip"]
ARCH = os.environ.get("EZSP_OFFLOAD_ARCH", "gfx950")

CFLAGS = [
    "-O3", "-std=c++17", "-fPIC", f"--offload-arch={ARCH}",
    "-ffp-contract=off", "-fno-fast-math",
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    "-Wall", "-Wno-unused-function", "-Wno-unused-result",
]


def hipcc() -> str:
    for cand in (os.environ.get("HIPCC"), "/opt/rocm/bin/hipcc",
                 shutil.which("hipcc")):
        if cand and os.path.exists(cand):
            return cand
    raise RuntimeError("hipcc not found (ROCm is required to build)")


def build(verbose: bool = False) -> str:
    """Compile every source (in parallel) and link libezsp.so; always runs."""
    cc = hipcc()
    os.makedirs(BUILD, exist_ok=True)
    procs, objs = [], []
    for src in SOURCES:
        obj = os.path.join(BUILD, src.replace(".hip", ".o"))
        cmd = [cc, *CFLAGS, "-c", os.path.join(CSRC, src), "-o", obj]
        if verbose:
            print(" ".join(cmd), flush=True)
        procs.append((src, subprocess.Popen(cmd, stdout=subprocess.PIPE,
                                            stderr=subprocess.STDOUT)))
        objs.append(obj)
    failed = []
    for src, p in procs:
        out, _ = p.communicate()
        text = out.decode(errors="replace")
        if p.returncode != 0:
            failed.append((src, text))
        elif verbose and text.strip():
            print(text, flush=True)
    if failed:
        msg = "\n".join(f"--- {s}\n{t}" for s, t in failed)
        raise RuntimeError("hipcc failed:\n" + msg)
    tmp = LIB + ".tmp%d" % os.getpid()
    cmd = [cc, "-shared", f"--offload-arch={ARCH}", *objs, "-o", tmp]
    if verbose:
        print(" ".join(cmd), flush=True)
    subprocess.check_call(cmd)
    os.replace(tmp, LIB)
    return LIB


if __name__ == "__main__":
    print(build(verbose="-v" in sys.argv))

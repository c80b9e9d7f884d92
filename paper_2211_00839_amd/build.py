"""Builds librcd.so (the HIP library behind the C ABI of include/rcd.h) for gfx950.

Run as ``python -m paper_2211_00839_amd.build``; hipcc cross-compiles without a GPU.
"""
from __future__ import annotations

import os
import subprocess
import sys

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "librcd.so")

HIPCC_FLAGS = [
    "-O3", "-std=c++17", "--offload-arch=gfx950", "-fPIC",
    # compiler-generated packed fp32 ops are kept out of every kernel
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    # no multiply and add is fused behind the source's back: every fused multiply-add in the kernels is
    # written as one (fmaf), so an expression gives the same bits in every kernel that evaluates it
    "-ffp-contract=off",
    "-Wno-unused-value",
]


# one object each, compiled side by side
SOURCES = ["rcd_lib.hip", "encoder_lib.hip"]


def build(verbose: bool = False) -> str:
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
    suffix = ".tmp.%d" % os.getpid()
    tmp = LIB + suffix
    objects = [os.path.join(HERE, src.replace(".hip", ".o")) + suffix for src in SOURCES]
    try:
        jobs = []
        for src, obj in zip(SOURCES, objects):
            cmd = [hipcc] + HIPCC_FLAGS + ["-c", os.path.join(CSRC, src), "-o", obj]
            if verbose:
                print(" ".join(cmd), flush=True)
            jobs.append(subprocess.Popen(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True))
        said = [job.communicate()[0] for job in jobs]
        failed = any(job.returncode != 0 for job in jobs)
        if not failed:
            cmd = [hipcc, "--offload-arch=gfx950", "-shared", "-fPIC"] + objects + ["-o", tmp]
            if verbose:
                print(" ".join(cmd), flush=True)
            res = subprocess.run(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
            said.append(res.stdout)
            failed = res.returncode != 0
        out = "\n".join(l for l in "".join(said).splitlines() if "packed-fp32-ops" not in l)
        if failed:
            raise RuntimeError("hipcc failed:\n" + out)
        if verbose and out.strip():
            print(out)
        os.replace(tmp, LIB)
    finally:
        for path in objects + [tmp]:
            if os.path.exists(path):
                os.remove(path)
    return LIB


if __name__ == "__main__":
    print(build(verbose=True))
    sys.exit(0)

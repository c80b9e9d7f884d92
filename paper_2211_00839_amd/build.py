"""Builds librcd.so (the HIP library behind the C ABI of include/rcd.h) for gfx950, and _encoder.so (the argument
marshalling of encoder.py, which calls it).

Run as ``python -m paper_2211_00839_amd.build``; hipcc cross-compiles without a GPU.  librcd.so needs nothing else; where a
host compiler, torch or a header of Python's is missing, _encoder.so is left out with a word, and encoder.py's calls raise.
"""
from __future__ import annotations

import os
import shutil
import subprocess
import sys
import sysconfig

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "librcd.so")
MARSHAL = os.path.join(HERE, "_encoder.so")

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
SOURCES = ["rcd_lib.hip", "encoder_lib.hip", "attention_lib.hip", "attention_backward_lib.hip"]


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
        _complain(any(job.returncode != 0 for job in jobs), said, verbose)
        _run([hipcc, "--offload-arch=gfx950", "-shared", "-fPIC"] + objects + ["-o", tmp], verbose)
        os.replace(tmp, LIB)
        missing = _missing_for_marshalling()
        if missing:
            if os.path.exists(MARSHAL):       # (of another build)
                os.remove(MARSHAL)
            print("_encoder.so is not built: %s" % missing, file=sys.stderr, flush=True)
        else:
            _run(_marshal_command(MARSHAL + suffix), verbose)
            os.replace(MARSHAL + suffix, MARSHAL)
    finally:
        for path in objects + [tmp, MARSHAL + suffix]:
            if os.path.exists(path):
                os.remove(path)
    return LIB


def _complain(failed, said, verbose):
    out = "\n".join(l for l in "".join(said).splitlines() if "packed-fp32-ops" not in l)
    if failed:
        raise RuntimeError("the compiler failed:\n" + out)
    if verbose and out.strip():
        print(out)


def _run(cmd, verbose):
    if verbose:
        print(" ".join(cmd), flush=True)
    res = subprocess.run(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
    _complain(res.returncode != 0, [res.stdout], verbose)


def _host_compiler():
    return os.environ.get("CXX", "g++")


def _missing_for_marshalling():
    """What _encoder.so cannot be built without and is not there, or None."""
    if not shutil.which(_host_compiler()):
        return "no host compiler %s" % _host_compiler()
    if not os.path.exists(os.path.join(sysconfig.get_path("include"), "Python.h")):
        return "no Python.h"
    try:
        import torch
    except ImportError as e:
        return "no torch (%s)" % e
    if not os.path.exists(os.path.join(os.path.dirname(os.path.abspath(torch.__file__)), "include", "ATen", "ATen.h")):
        return "no headers of torch"
    return None


def _marshal_command(out):
    """Host code alone, against torch's headers and the library just built."""
    import torch

    root = os.path.dirname(os.path.abspath(torch.__file__))
    return [_host_compiler(), "-O2", "-std=c++17", "-fPIC", "-shared", "-w", "-I", os.path.join(root, "include"),
            "-I", os.path.join(root, "include", "torch", "csrc", "api", "include"), "-I", sysconfig.get_path("include"),
            os.path.join(CSRC, "encoder_marshal.cpp"), "-o", out, "-L", os.path.join(root, "lib"), "-ltorch_python", "-ltorch_cpu",
            "-ltorch", "-lc10", "-L", HERE, "-lrcd", "-Wl,-rpath,$ORIGIN"]


if __name__ == "__main__":
    print(build(verbose=True))
    sys.exit(0)

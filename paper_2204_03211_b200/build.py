"""Builds the C-ABI shared library in-tree with nvcc for sm_100a.

    python -m paper_2204_03211_b200.build [--force] [--verbose]

The library, and the small Python extension that calls it (csrc/ps_python.c, gcc),
are rebuilt when any source under csrc/ or the public header is newer than them.  FMA contraction is disabled (--fmad=false) on top of the
explicit round-to-nearest intrinsics in the kernels; fast-math is never used.
"""
import glob
import os
import subprocess
import sys
import sysconfig

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libps_b200.so")
OPS = os.path.join(HERE, "_ops" + sysconfig.get_config_var("EXT_SUFFIX"))
SOURCES = [os.path.join(CSRC, "ps_service.cu"), os.path.join(CSRC, "ps_planner.cpp"), os.path.join(CSRC, "ps_peer.cpp"),
           os.path.join(CSRC, "ps_mx.cu"), os.path.join(CSRC, "ps_clip.cu"),
           os.path.join(CSRC, "ps_ortho.cu"), os.path.join(CSRC, "ps_xent.cu")]


def _deps():
    return (glob.glob(os.path.join(CSRC, "*")) + glob.glob(os.path.join(ROOT, "include", "*.h")))


def nvcc_command(verbose: bool = False):
    cmd = ["nvcc", "-std=c++17", "-O3", "-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo",
           "--fmad=false", "-Xcompiler", "-fPIC,-Wall,-O2", "-shared", "-cudart", "shared",
           "-I", os.path.join(ROOT, "include"), "-o", LIB] + SOURCES
    if verbose:
        cmd.insert(1, "-Xptxas")
        cmd.insert(2, "-v")
    return cmd


def ops_command():
    return ["gcc", "-std=gnu11", "-O2", "-Wall", "-fPIC", "-shared", "-I", sysconfig.get_paths()["include"],
            "-I", os.path.join(ROOT, "include"), "-o", OPS, os.path.join(CSRC, "ps_python.c"), "-L", HERE, "-lps_b200",
            "-Wl,-rpath,$ORIGIN"]


def _run(cmd, target: str, verbose: bool):
    res = subprocess.run(cmd, capture_output=True, text=True)
    if verbose or res.returncode:
        sys.stderr.write(res.stdout + res.stderr)
    if res.returncode:
        raise RuntimeError("%s failed building %s" % (cmd[0], target))


def build(force: bool = False, verbose: bool = False) -> str:
    newest = max(os.path.getmtime(p) for p in _deps())
    if force or not os.path.exists(LIB) or os.path.getmtime(LIB) < newest:
        _run(nvcc_command(verbose), LIB, verbose)
    if force or not os.path.exists(OPS) or os.path.getmtime(OPS) < newest:
        _run(ops_command(), OPS, verbose)
    return LIB


if __name__ == "__main__":
    print(build(force="--force" in sys.argv, verbose="--verbose" in sys.argv))

"""Builds libw2v.so (HIP, gfx950) in-tree next to this file.

hipcc compiles the device translation units for gfx950 only; the host-only
table builder is compiled by g++. The shared library exports the C ABI of
include/w2v.h and nothing that depends on torch.
"""
import os
import subprocess
import sys
from concurrent.futures import ThreadPoolExecutor

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(HERE, "csrc")
BUILD = os.path.join(HERE, "_build")
LIB = os.path.join(HERE, "libw2v.so")
MEASURE_LIB = os.path.join(HERE, "libw2v_measure.so")
HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")

HIP_SOURCES = ["api.hip", "epoch_kernels.hip", "pairwise_kernels.hip",
               "step_kernels.hip", "step_sorted.hip", "vocab.hip", "radix_sort.hip",
               "head_api.hip", "linear.hip", "linear_f32.hip", "linear_bf16.hip",
               "linear_f16.hip", "distill.hip", "sample.hip", "ends_api.hip",
               "embed.hip", "dropout.hip", "linear_q4.hip", "beam.hip"]
CXX_SOURCES = ["tables.cpp"]

HIP_FLAGS = [
    "-O3", "--offload-arch=gfx950", "-fPIC", "-std=c++17",
    "-munsafe-fp-atomics",
    # keep the compiler from emitting packed fp32 arithmetic
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    "-I" + os.path.join(ROOT, "include"), "-Wall", "-Wno-unused-function",
]
CXX_FLAGS = ["-O2", "-fPIC", "-std=c++17", "-ffp-contract=off",
             "-fno-fast-math", "-Wall", "-I" + os.path.join(ROOT, "include")]


def _run(cmd, verbose):
    if verbose:
        print(" ".join(cmd), flush=True)
    r = subprocess.run(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT,
                       text=True)
    out = "\n".join(l for l in r.stdout.splitlines()
                    if "packed-fp32-ops" not in l and "not a recognized feature" not in l)
    if r.returncode != 0:
        raise RuntimeError(f"build step failed ({r.returncode}):\n{' '.join(cmd)}\n{out}")
    if verbose and out.strip():
        print(out)


def build(verbose: bool = False, jobs: int = 8) -> str:
    os.makedirs(BUILD, exist_ok=True)
    cmds, objs = [], []
    for src in HIP_SOURCES:
        obj = os.path.join(BUILD, src + ".o")
        objs.append(obj)
        cmds.append([HIPCC, *HIP_FLAGS, "-c", os.path.join(CSRC, src), "-o", obj])
    for src in CXX_SOURCES:
        obj = os.path.join(BUILD, src + ".o")
        objs.append(obj)
        cmds.append(["g++", *CXX_FLAGS, "-c", os.path.join(CSRC, src), "-o", obj])
    mobj = os.path.join(BUILD, "row_rmw.hip.o")
    cmds.append([HIPCC, *HIP_FLAGS, "-c", os.path.join(HERE, "measure", "row_rmw.hip"),
                 "-o", mobj])
    with ThreadPoolExecutor(max_workers=jobs) as ex:
        list(ex.map(lambda c: _run(c, verbose), cmds))
    tmp = LIB + ".tmp"
    _run([HIPCC, "--offload-arch=gfx950", "-shared", "-fPIC", "-o", tmp, *objs],
         verbose)
    os.replace(tmp, LIB)
    # the memory-ceiling measurement kernel of bench.py, kept out of libw2v
    mtmp = MEASURE_LIB + ".tmp"
    _run([HIPCC, "--offload-arch=gfx950", "-shared", "-fPIC", "-o", mtmp, mobj], verbose)
    os.replace(mtmp, MEASURE_LIB)
    return LIB


if __name__ == "__main__":
    print(build(verbose="-v" in sys.argv))

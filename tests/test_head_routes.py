"""Which tile, split and copy the products of head_shapes.py get: csrc's own
plan, compiled for the host (no GPU)."""
import os
import shutil
import subprocess

import pytest

import head_shapes as shapes

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
SOURCE = r"""
#include <cstdio>
#include <cstdlib>
#include "linear_plan.h"
using namespace w2v;
int main(int argc, char** argv) {
  for (int i = 1; i + 4 <= argc; i += 4) {
    const int M = atoi(argv[i]), N = atoi(argv[i + 1]), K = atoi(argv[i + 2]);
    const int type = atoi(argv[i + 3]);
    const Plan f = plan_product(M, N, K, type, false);
    const BackwardPlan b = plan_backward(M, N, K, type, W2V_ACTIVATION_NONE);
    printf("%d %d %d %d %d %d %d %d %d\n", few_rows(M, K), f.tile, f.splits > 1,
           copy_bytes(M, M, N, K, type) > 0, b.dx.tile, b.dx.splits > 1, b.dw.tile,
           b.dw.splits > 1, b.x > 0);
  }
}
"""
TYPES = {shapes.F32: 0, shapes.BF16: 1, shapes.F16: 2}


@pytest.mark.skipif(shutil.which("g++") is None or not os.path.isdir("/opt/rocm/include"),
                    reason="needs g++ and HIP's headers")
def test_large_products_take_the_kernels_that_are_tested(tmp_path):
    source, exe = tmp_path / "plan.cpp", str(tmp_path / "plan")
    source.write_text(SOURCE)
    r = subprocess.run(
        ["g++", "-std=c++17", "-O1", "-D__HIP_PLATFORM_AMD__", "-I/opt/rocm/include",
         "-I" + os.path.join(ROOT, "include"),
         "-I" + os.path.join(ROOT, "paper_1611_06172_amd", "csrc"), str(source), "-o", exe],
        capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stderr
    keys = list(shapes.FORWARD) + list(shapes.BACKWARD)
    args = [str(v) for M, N, K, t in keys for v in (M, N, K, TYPES[t])]
    out = subprocess.run([exe, *args], capture_output=True, text=True, timeout=60)
    rows = [[int(v) for v in line.split()] for line in out.stdout.splitlines()]
    assert len(rows) == len(keys)
    for key, row in zip(keys, rows):
        few, tile, split, copied = row[:4]
        if key in shapes.FORWARD:
            assert not few and (tile, bool(split), bool(copied)) == shapes.FORWARD[key], key
        if key in shapes.BACKWARD:
            want = shapes.BACKWARD[key]
            assert tuple(row[4:]) == tuple(int(v) for v in want), key

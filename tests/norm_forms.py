"""Shapes that reach every form of the RMS norm's kernels, and the plan the library makes for a shape."""
import subprocess
import tempfile
from pathlib import Path

from paper_2504_06881_b200 import build

# (N, C, P): each makes a block (P = 1: a warp) of the backward pass go over three tiles (rows) or more
MANY = [(1300, 20, 17), (1300, 20, 8), (1300, 20, 4), (650, 33, 33), (650, 30, 40), (1300, 60, 12), (1300, 100, 8), (700, 100, 4), (700, 100, 7),
        (700, 130, 16), (350, 200, 12), (700, 200, 9), (330, 300, 24), (330, 300, 20), (330, 300, 13), (340, 512, 8),
        (330, 512, 12), (300, 512, 7), (620, 513, 7), (310, 516, 40), (610, 520, 20), (10, 33, 4099), (24, 64, 1600),
        (2500, 64, 1), (2500, 200, 1), (2500, 400, 1), (3600, 33, 1), (3600, 250, 1), (3700, 300, 1), (2500, 700, 1), (3600, 511, 1), (3600, 1021, 1), (2500, 1024, 1)]
# few tiles, and the kernels that go over channels in groups: rows of more than 1024 channels, sums beyond shared memory
FEW = [(2, 513, 1), (3, 1025, 1), (2, 1028, 1), (2, 4096, 1), (700, 1100, 1), (1300, 1028, 1), (3, 24, 12), (2, 100, 28), (2, 300, 196), (2, 200, 49),
       (1, 9001, 40), (1, 9001, 33), (3, 9004, 12), (300, 8193, 3)]

MAIN = """
#include <cstdio>
#include "tconv.h"
#include "tconv_norm.cuh"
using namespace tconv;
int main() {
    NormArgs a{};
    long long P;
    int dtype;
    while (scanf("%d %d %lld %d", &a.N, &a.C, &P, &dtype) == 4) {
        a.P = P;
        const NormPlan p = plan_norm(a, dtype);
        printf("%d %d %d %d\\n", p.vec, p.form, p.blocks, p.parts);
    }
}
"""


def plans(shapes):
    """[(vec, form, blocks, parts)] of (N, C, P, "f32" or "bf16")."""
    with tempfile.TemporaryDirectory() as tmp:
        src, exe = Path(tmp) / "plan.cu", Path(tmp) / "plan"
        src.write_text(MAIN)
        subprocess.run(build._nvcc_base(False, "c++20") + ["-o", str(exe), str(src)], check=True, capture_output=True)
        lines = "\n".join(f"{n} {c} {p} {0 if d == 'f32' else 1}" for n, c, p, d in shapes)
        out = subprocess.run([str(exe)], input=lines, check=True, capture_output=True, text=True).stdout
    return [tuple(map(int, line.split())) for line in out.splitlines()]

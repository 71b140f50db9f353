"""Which kernel csrc/linear_plan.h takes for a product of 16-bit matrices, asked of the header itself on the host."""
import os
import subprocess
import tempfile

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
KERNELS = {0: "256", 1: "128", 2: "64", 3: "128 deep", 4: "few", 5: "64 twice", -1: "any", -2: "any few"}
FORMS = {"kk": 0, "kn": 1, "nn": 2}
ENDS = {"store": 0, "gated": 1, "gated_grad": 2, "scores": 3, "scores_grad": 4}

SOURCE = """
#include <stdio.h>
#include "linear_plan.h"
int main(int argc, char **)
{
    long long v[10];
    for (;;) {
        for (int i = 0; i < (argc > 1 ? 10 : 7); ++i)
            if (scanf("%lld", &v[i]) != 1) return 0;
        if (argc > 1) {
            const mg::LinearSize sizes[3] = {{v[0], v[1], v[2]}, {v[3], v[4], v[5]}, {v[6], v[7], v[8]}};
            const mg::LinearPlan how = mg::linear_plan_together(sizes, static_cast<size_t>(v[9]));
            printf("%d %d %d\\n", how.tile, how.slices, how.k_per_slice);
            continue;
        }
        const mg::LinearPlan how = mg::linear_plan(static_cast<int>(v[0]), static_cast<int>(v[1]), v[2], v[3], v[4], v[5] != 0, static_cast<size_t>(v[6]));
        printf("%d %d %d\\n", how.tile, how.slices, how.k_per_slice);
    }
}
"""


def choices(problems):
    """(kernel, slices, values of the sum in a slice) of each problem: (form, end, rows, cols, k[, aligned[, room]])"""
    lines = []
    for form, end, rows, cols, k, *more in problems:
        aligned, room = (more + [True, 1 << 40][len(more):])
        lines.append(f"{FORMS[form]} {ENDS[end]} {rows} {cols} {k} {int(aligned)} {room}")
    return asked(lines)


def together(problems):
    """the same of products that may go in one launch: (rows, cols, k) of the first, with its operand across the sum, and of two more; "any": one by one"""
    return asked([" ".join(str(v) for size in sizes for v in size) + f" {room}" for *sizes, room in problems], "together")


def asked(lines, *mode):
    with tempfile.TemporaryDirectory() as folder:
        source, program = os.path.join(folder, "ask.cpp"), os.path.join(folder, "ask")
        with open(source, "w") as f:
            f.write(SOURCE)
        subprocess.run(["g++", "-O1", "-std=c++17", "-D__HIP_PLATFORM_AMD__", "-I", os.path.join(ROOT, "paper_1705_05249_amd", "csrc"), "-I", "/opt/rocm/include", source, "-o", program],
                       check=True)
        out = subprocess.run([program, *mode], input="\n".join(lines) + "\n", check=True, capture_output=True, text=True).stdout
    answers = [tuple(int(x) for x in line.split()) for line in out.splitlines()]
    assert len(answers) == len(lines)
    return [(KERNELS[tile], slices, each) for tile, slices, each in answers]

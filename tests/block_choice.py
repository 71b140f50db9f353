"""Which kernel csrc/block_plan.h takes for a product of 8-bit matrices, asked of the header itself on the host."""
import os
import subprocess
import tempfile

from paper_1705_05249_amd import experts as X

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
KERNELS = {0: "256", 1: "128", 2: "64", -1: "any 128", -2: "any 64", -3: "few"}
MODES = {"dense": 0, "rows": 1, "sum": 2}

SOURCE = """
#include <stdio.h>
#include "block_plan.h"
int main()
{
    long long v[20];
    for (;;) {
        for (long long &x : v)
            if (scanf("%lld", &x) != 1) return 0;
        mg::BlockProblem p{};
        p.mode = static_cast<int>(v[0]);
        p.groups = mg::Groups{nullptr, static_cast<int>(v[1]), v[2], v[18] ? reinterpret_cast<const int32_t *>(64) : nullptr, static_cast<int>(v[19])};
        p.m = v[2]; p.n = v[3]; p.k = v[4];
        p.pow2 = v[5]; p.fp32_sums = v[6]; p.a_square = v[7]; p.b_square = v[8];
        p.A = reinterpret_cast<const uint8_t *>(v[9]); p.lda = v[10]; p.ldsa = v[11];
        p.B = reinterpret_cast<const uint8_t *>(v[12]); p.ldb = v[13]; p.ldsb = v[14];
        p.stride_b = v[15];
        p.workspace = reinterpret_cast<void *>(v[16]); p.workspace_bytes = static_cast<size_t>(v[17]);
        const mg::Plan how = mg::plan(p);
        printf("%d %d %d %d %d\\n", how.tile, mg::block_sums(p), how.slices, how.fragments, how.few_b);
    }
}
"""


def choices(problems):
    """(kernel, kind of sums, slices, fragments) of each; a problem is a dict: mode, m, n, k and what differs from the ordinary"""
    lines = []
    for p in problems:
        k, mode = p["k"], MODES[p.get("mode", "dense")]
        groups, fan = p.get("groups", 0 if mode == 0 else 1), p.get("fan", 1)
        along = k if mode != 2 else X.mg_grouped_columns(k, groups)
        lda, ldb = p.get("lda", -(-along // 16) * 16), p.get("ldb", -(-along // 16) * 16)
        blocks = -(-along // 128)
        lines.append((mode, groups, p["m"], p["n"], k, p.get("pow2", False), p.get("fp32", False), p.get("a_square", False), p.get("b_square", False),
                      4096 + p.get("start", 0), lda, blocks, 8192, ldb, blocks, p["n"] * ldb, 4096 if p.get("workspace", 0) else 0, p.get("workspace", 0),
                      p.get("indexed", False), fan))
    with tempfile.TemporaryDirectory() as folder:
        source, program = os.path.join(folder, "choice.cpp"), os.path.join(folder, "choice")
        with open(source, "w") as f:
            f.write(SOURCE)
        subprocess.run(["g++", "-std=c++17", "-O1", "-D__HIP_PLATFORM_AMD__", "-I/opt/rocm/include", "-I", os.path.join(ROOT, "paper_1705_05249_amd", "csrc"), source, "-o", program],
                       check=True)
        text = "\n".join(" ".join(str(int(v)) for v in line) for line in lines)
        out = subprocess.run([program], input=text, capture_output=True, text=True, check=True, timeout=60).stdout.split("\n")
    result = []
    for line in out[:len(lines)]:
        tile, sums, slices, fragments, _ = (int(v) for v in line.split())
        result.append((KERNELS[tile], ("pow2", "any", "fp32", "square", "fp32 pow2")[sums], slices, fragments))
    return result

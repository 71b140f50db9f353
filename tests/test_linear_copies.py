"""Which launches a copy of many rows is made of (csrc/layers.h), asked of the header itself on the host: a launch counts pieces in 32 bits."""
import os
import subprocess

import pytest

from paper_1705_05249_amd import layers as L

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
SOURCE = """
#include <stdio.h>
#include "layers.h"
int main()
{
    long long rows, cols, ld;
    while (scanf("%lld %lld %lld", &rows, &cols, &ld) == 3) {
        mg::LinearCopies c{};
        c.from[0] = reinterpret_cast<const void *>(uintptr_t(1) << 40);
        c.to[0] = reinterpret_cast<void *>(uintptr_t(1) << 44);
        c.targets = reinterpret_cast<const int64_t *>(uintptr_t(1) << 30);
        c.weights = reinterpret_cast<const float *>(uintptr_t(1) << 20);
        c.count = 1; c.rows[0] = rows; c.cols[0] = static_cast<int>(cols); c.ld[0] = ld;
        auto tell = [](const mg::LinearCopies &p) {
            printf("%lld %lld %lld %lld %lld\\n", (long long)p.rows[0], (long long)reinterpret_cast<uintptr_t>(p.from[0]), (long long)reinterpret_cast<uintptr_t>(p.to[0]),
                   (long long)reinterpret_cast<uintptr_t>(p.targets), (long long)reinterpret_cast<uintptr_t>(p.weights));
        };
        while (c.rows[0] > mg::copy_rows(cols)) tell(mg::take_copy_rows(c, mg::copy_rows(cols)));
        tell(c);
        printf("end\\n");
    }
}
"""


def padded(v):
    return -(-v // 64) * 64


@pytest.fixture(scope="module")
def parts(tmp_path_factory):
    folder = tmp_path_factory.mktemp("copies")
    source, program = folder / "ask.cpp", folder / "ask"
    source.write_text(SOURCE)
    subprocess.run(["g++", "-O1", "-std=c++17", "-D__HIP_PLATFORM_AMD__", "-I", os.path.join(ROOT, "paper_1705_05249_amd", "csrc"), "-I", "/opt/rocm/include", str(source), "-o", str(program)],
                   check=True)

    def ask(rows, cols, ld):
        out = subprocess.run([str(program)], input=f"{rows} {cols} {ld}\n", check=True, capture_output=True, text=True).stdout.splitlines()
        assert out.pop() == "end"
        return [tuple(int(v) for v in line.split()) for line in out]
    return ask


# tokens, width of FP32 matrices that the gradient of the loss accepts: units of 16 bits
FP32 = [(16_760_000, 1025), ((1 << 24) - 1, 1024), ((1 << 24) - 1, 993), (4_100_000, 4190), (1, (1 << 24) - 1), (1025, (1 << 24) - 1), (1 << 20, 1 << 14), (1000, 1), (300, 1001)]


@pytest.mark.parametrize("tokens,width", FP32)
def test_parts_cover_the_rows_and_fit_a_launch(tokens, width, parts):
    if tokens * width <= 1 << 34 and tokens < 1 << 24:
        assert L.mg_vocab_loss_grad_workspace_bytes(L.MG_F32, tokens, width, 8) > 0             # a size that the call accepts
    cols, ld = 2 * width, 2 * width + 6
    done = 0
    for rows, source, to, targets, weights in parts(tokens, cols, ld):
        pieces = rows * (padded(cols) // 8)
        assert rows > 0 and -(-pieces // 256) * 256 <= 1 << 32
        assert source == (1 << 40) + done * ld * 2 and to == (1 << 44) + done * padded(cols) * 2 and targets == (1 << 30) + done * 8 and weights == (1 << 20) + done * 4
        done += rows
    assert done == tokens


def test_matrices_of_16_bits_go_in_one_launch(parts):
    """2^34 elements at most, fewer than 2^24 rows or columns"""
    for rows, cols in (((1 << 24) - 1, 1024), ((1 << 24) - 1, 1), (1 << 10, (1 << 24) - 1), (16_000_000, 1073), (1 << 17, 1 << 17), (1, 1), (5, 0)):
        assert rows * cols <= 1 << 34 and len(parts(rows, cols, cols)) == 1
    assert len(parts(16_760_000, 2050, 2050)) == 2

"""The kernels of the 8-bit products that are built: those that some call reaches, each once, and no other; and of those that read LDS by hand-waited instructions every single
one is looked over (see test_reads_in_flight.py)."""
import re
import struct

from paper_1705_05249_amd import gemm as G
from tests import test_reads_in_flight as T

POW2, ANY, FP32, SQUARE, FP32_POW2 = range(5)
DENSE, ROWS, SUM = range(3)
NAME = re.compile(rb"_ZN2mg(?:12_GLOBAL__N_1)?16block_(dma|any|few)_kernelI([\w]+?)EEvNS_?\w*?Args")


def code_objects():
    data, at = open(G.LIB_PATH, "rb").read(), 0
    while (at := data.find(T.MAGIC, at)) >= 0:
        p = at + len(T.MAGIC) + 8
        for _ in range(struct.unpack_from("<Q", data, at + len(T.MAGIC))[0]):
            offset, size, length = struct.unpack_from("<QQQ", data, p)
            target, p = data[p + 24: p + 24 + length], p + 24 + length
            if b"gfx950" in target:
                yield data[at + offset: at + offset + size]
        at += 1


def built(kind):
    """template arguments of the kernels of a kind"""
    found = set()
    for code in code_objects():
        for name, arguments in NAME.findall(code):
            if name.decode() == kind:
                found.add(tuple(int(v) for v in re.findall(rb"Li(\d+)E?", arguments)) + ((b"Fp8Fragment" in arguments,) if kind == "few" else ()))
    return found


def dma():
    """mode, sums, tile, wavefronts down and across, stages: SUMS_SQUARE (one scale for 128 rows of B) is for large tiles of operands that have such blocks"""
    wanted = set()
    for mode in (DENSE, ROWS, SUM):
        for sums in (POW2, ANY, FP32, FP32_POW2) + ((SQUARE,) if mode != SUM else ()):
            fp32 = sums in (FP32, FP32_POW2)
            wanted.add((mode, sums, 256, 128 if fp32 else 256, *((4, 2) if fp32 or sums == ANY else (2, 4)), 2))
            if sums != SQUARE:
                wanted |= {(mode, sums, 128, 128, 2, 2, 2), (mode, sums, 64, 64, 2, 2, 4)}
    return wanted


def test_kernels_of_aligned_operands():
    assert built("dma") == dma()


def test_kernels_of_any_address_and_of_few_rows():
    assert built("any") == {(mode, sums, size) for mode in (DENSE, ROWS, SUM) for sums in (POW2, ANY, FP32) for size in (64, 128)}
    # (rows of experts: 16 for an expert at most, two fragments only for up to 32 rows of one product)
    assert built("few") == {(mode, waves, fragments, fp8) for mode in (DENSE, ROWS) for waves in (4, 8) for fragments in ((1, 2) if mode == DENSE else (1,)) for fp8 in (False, True)}


def test_every_hand_waited_kernel_is_looked_over(tmp_path, monkeypatch):
    monkeypatch.setattr(T, "KERNEL", re.compile(r"^[0-9a-f]+ <(_ZN2mg16block_dma_kernelI\w+EvNS_9BlockArgsE)>:$"))
    seen, wrong = set(), {}
    for n, code in enumerate(code_objects()):
        if b"block_dma_kernel" not in code:
            continue
        path = tmp_path / f"{n}.co"
        path.write_bytes(code)
        for name, body in T.kernels(str(path)):
            reads, touched = T.touched_in_flight(body)
            if reads > 0:
                seen.add(tuple(int(v) for v in re.findall(r"Li(\d+)E", name)))
            if touched:
                wrong[name] = sorted(touched)[:4]
    assert seen == dma()
    assert not wrong, wrong

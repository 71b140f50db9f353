"""The direct-to-LDS kernels of the dense layers that are built: those that some call reaches, each once; none touches a register that an LDS read is still to
write (see test_reads_in_flight.py)."""
import re
import struct

import pytest

from paper_1705_05249_amd import gemm as G
from tests import test_reads_in_flight as T

KK, KN, NN = range(3)
STORE, GATED, GATED_GRAD, SCORES, SCORES_GRAD = range(5)
NAME = re.compile(rb"_ZN2mg(?:12_GLOBAL__N_1)?1[67]linear_(dma|any|pp)_kernelI([\w]+?)EEvNS_?\w*?Args")
PAIRS = {(KK, STORE), (KK, GATED), (KK, SCORES), (KK, SCORES_GRAD), (KN, STORE), (KN, GATED_GRAD), (NN, STORE)}


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
    """(bfloat16, numbers) of the kernels of a kind"""
    found = set()
    for code in code_objects():
        for name, arguments in NAME.findall(code):
            if name.decode() == kind:
                found.add((arguments.startswith(b"DF16b"), *(int(v) for v in re.findall(rb"L[ib](\d+)E?", arguments))))
    return found


def dma():
    tiles = {(128, 128, 2, 2, 2, 1), (128, 128, 2, 2, 4, 1), (64, 64, 2, 2, 4, 1), (64, 64, 2, 2, 4, 2)}
    return {(kind, *pair, *tile) for kind in (False, True) for pair in PAIRS for tile in tiles}


def pp():
    """the 256 x 256 tile; what a block keeps, or dz, passes the caches by or does not"""
    return {(kind, *pair, past) for kind in (False, True) for pair in PAIRS for past in (0, 1) if not past or pair in ((KK, GATED), (KN, GATED_GRAD), (KK, SCORES_GRAD))}


def test_kernels_that_are_built():
    assert built("dma") == dma()
    assert built("pp") == pp()
    assert built("any") == {(kind, *pair) for kind in (False, True) for pair in PAIRS}


def few():
    """bfloat16, end, blocks of 16 columns and rows, wavefronts, stages, weights pass the caches by"""
    kernels = {(STORE, 1, 1, 8, 4), (STORE, 1, 2, 8, 3), (GATED, 2, 1, 4, 2), (GATED, 2, 2, 4, 3), (SCORES, 4, 1, 4, 2), (SCORES, 4, 2, 4, 3)}
    return {(kind, *kernel, once) for kind in (False, True) for kernel in kernels for once in (0, 1)}


def together():
    """bfloat16, tile, stages"""
    return {(kind, *kernel) for kind in (False, True) for kernel in ((128, 2), (64, 4))}


@pytest.mark.parametrize("start,wanted", [("_ZN2mg17linear_dma_kernelI", dma), ("_ZN2mg16linear_pp_kernelI", pp), ("_ZN2mg12_GLOBAL__N_121linear_few_dma_kernelI", few),
                                          ("_ZN2mg12_GLOBAL__N_122linear_together_kernelI", together)])
def test_every_hand_waited_kernel_is_looked_over(tmp_path, monkeypatch, start, wanted):
    monkeypatch.setattr(T, "KERNEL", re.compile(r"^[0-9a-f]+ <(" + start + r"\w+E+vNS\w*?1[04]Linear(?:Args|Together)E)>:$"))
    seen, wrong = set(), {}
    for n, code in enumerate(code_objects()):
        if start.encode() not in code:
            continue
        path = tmp_path / f"{n}.co"
        path.write_bytes(code)
        for name, body in T.kernels(str(path)):
            reads, touched = T.touched_in_flight(body)
            if reads > 0:
                seen.add((name.startswith(start + "DF16b"), *(int(v) for v in re.findall(r"L[ib](\d+)E", name))))
            if touched:
                wrong[name] = sorted(touched)[:4]
    assert seen == wanted()
    assert not wrong, wrong

"""As test_reads_in_flight.py, for the kernels of block_dma_kernel.h: no instruction touches a register that an LDS read is still to write."""
import re
import struct

from paper_1705_05249_amd import gemm as G
from tests import test_reads_in_flight as T


def test_no_register_is_touched_while_a_read_may_write_it(tmp_path, monkeypatch):
    monkeypatch.setattr(T, "KERNEL", re.compile(r"^[0-9a-f]+ <(_ZN2mg16block_dma_kernelI\w+EvNS_9BlockArgsE)>:$"))
    data, at, seen, wrong = open(G.LIB_PATH, "rb").read(), 0, 0, {}
    while (at := data.find(T.MAGIC, at)) >= 0:
        p = at + len(T.MAGIC) + 8
        for _ in range(struct.unpack_from("<Q", data, at + len(T.MAGIC))[0]):
            offset, size, length = struct.unpack_from("<QQQ", data, p)
            target, p = data[p + 24: p + 24 + length], p + 24 + length
            code = data[at + offset: at + offset + size]
            if b"gfx950" in target and b"block_dma_kernel" in code:
                path = tmp_path / f"{at}.co"
                path.write_bytes(code)
                for name, body in T.kernels(str(path)):
                    reads, touched = T.touched_in_flight(body)
                    seen += reads > 0
                    if touched:
                        wrong[name] = sorted(touched)[:4]
        at += 1
    assert seen >= 18, seen
    assert not wrong, wrong

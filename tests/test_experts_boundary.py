"""Host-side checks of include/mg_experts.h that need no GPU: symbols, every refusal, sizes, and that arguments arrive."""
import ctypes
import os
import re

import pytest

from paper_1705_05249_amd import experts as X, gemm as G

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
FAKE = 0x1000          # never dereferenced: every call below fails validation or returns early
ROW, COL = X.MG_ROW_MAJOR, X.MG_COL_MAJOR


def test_header_symbols_are_exported():
    text = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "mg_experts.h")).read(), flags=re.S)
    assert sorted(set(re.findall(r"\b(mg_[a-z0-9_]+)\s*\(", text))) == sorted(X.EXPORTS)
    for name in X.EXPORTS:
        assert getattr(X.lib(), name) is not None
    assert all(G.status_string(code) != "unknown status" for code in range(-20, -24, -1)) and G.status_string(-24) == "unknown status"


def test_every_argument_arrives():
    import torch
    L, call = X.lib(), X._native()
    try:
        for name in X._calls:
            types, seen, args, expected = getattr(L, name).argtypes, [], [], []
            for i, t in enumerate(types):
                if t is ctypes.c_size_t:
                    expected.append(args[-1].numel() * args[-1].element_size())
                elif t is ctypes.c_float:
                    args.append(0.5 + i)
                    expected.append(0.5 + i)
                elif t is ctypes.c_void_p and i + 1 < len(types):
                    args.append(torch.zeros(3 + i, dtype=torch.float32))
                    expected.append(args[-1].data_ptr())
                else:
                    args.append((1 << 40) + i if t is ctypes.c_int64 else 1000 + i)
                    expected.append(args[-1])
            made = ctypes.CFUNCTYPE(ctypes.c_int32, *types)(lambda *a: seen.extend(a) or -7)
            call.bind({name: ctypes.cast(made, ctypes.c_void_p).value}, G._stream_calls, G._by_ctypes)
            assert getattr(call, name)(*args) == -7
            assert seen == expected, name
            seen.clear()
            assert getattr(X, name)(*args, check=False) == -7          # the function of the module hands all of them on, in this order
            assert seen == expected, name
    finally:
        X._call = None
        X._native()


def quantize(dtype=X.MG_F32, block=X.MG_BLOCK_ROW, rows=4, cols=200, X_=FAKE, ldx=200, Q=FAKE, ldq=200, S=FAKE, lds=2, T=FAKE, ldt=4, ST=FAKE, ldst=1):
    return X.mg_block_quantize(dtype, block, rows, cols, X_, ldx, Q, ldq, S, lds, T, ldt, ST, ldst, stream=0, check=False)


def test_quantize_refusals():
    assert quantize(rows=-1) == -4 and quantize(cols=-1) == -4 and quantize(rows=1 << 31) == -4
    assert quantize(rows=1 << 30, cols=1 << 20, ldx=1 << 20, ldq=1 << 20, ldt=1 << 30, lds=1 << 13, ldst=1 << 23) == -4
    assert quantize(ldx=199) == -5 and quantize(ldq=199) == -6 and quantize(ldt=3) == -7
    assert quantize(X_=None) == -8 and quantize(Q=None) == -8 and quantize(S=None) == -8 and quantize(T=None) == -8 and quantize(ST=None) == -8
    assert quantize(Q=None, S=None, T=None, ST=None) == -8
    assert quantize(dtype=3) == -20 and quantize(dtype=-1) == -20
    assert quantize(block=0) == -21
    assert quantize(lds=1) == -23 and quantize(ldst=0) == -23
    assert quantize(rows=0, X_=None) == 0 and quantize(cols=0, X_=None, lds=1) == 0
    assert quantize(rows=0, ldx=100) == -5                          # leading dimensions are checked all the same


def test_quantize_batched_refusals():
    def call(batch=2, sx=800, sq=800, ss=8, st=800, sst=200):
        return X.mg_block_quantize_batched(X.MG_F16, X.MG_BLOCK_ROW, batch, 4, 200, FAKE, 200, sx, FAKE, 200, sq, FAKE, 2, ss, FAKE, 4, st, FAKE, 1, sst, stream=0,
                                           check=False)
    assert call(batch=-1) == -9 and call(batch=65536) == -9 and call(batch=0) == 0
    for name in ("sx", "sq", "ss", "st", "sst"):
        assert call(**{name: -1}) == -14


def test_quantize_grouped_refusals():
    def call(groups=3, offsets=FAKE, rows=100, fan=2, source=FAKE, ldt=512, ldst=4, dtype=X.MG_BF16, lds=1, cols=64):
        return X.mg_block_quantize_grouped(dtype, groups, offsets, rows, cols, FAKE, 64, source, fan, FAKE, 64, FAKE, lds, FAKE, ldt, FAKE, ldst, stream=0, check=False)
    assert X.mg_grouped_columns(100, 3) == 512 and X.mg_grouped_columns(128, 1) == 256 and X.mg_grouped_columns(0, 2) == 256
    assert X.mg_grouped_columns(-1, 2) == -1 and X.mg_grouped_columns(5, 0) == -1 and X.mg_grouped_columns(5, 1025) == -1
    assert call(ldt=511) == -7 and call(ldst=3) == -23
    assert call(groups=0) == -22 and call(groups=1025) == -22 and call(fan=0) == -22 and call(fan=65) == -22
    assert call(groups=0, dtype=9) == -20
    assert call(offsets=None) == -8
    assert call(rows=0, offsets=None) == 0


def product(layout=ROW, m=5, n=6, k=300, alpha=1.0, scales=X.MG_SCALES_ANY, a_block=X.MG_BLOCK_ROW, A=FAKE, lda=300, SA=FAKE, ldsa=3,
            b_block=X.MG_BLOCK_SQUARE, B=FAKE, ldb=300, SB=FAKE, ldsb=3, beta=0.0, c_type=X.MG_BF16, C=FAKE, ldc=6, ws=None):
    return X.mg_block_gemm(layout, m, n, k, alpha, scales, a_block, A, lda, SA, ldsa, b_block, B, ldb, SB, ldsb, beta, c_type, C, ldc, ws, 0, check=False)


def test_product_refusals():
    assert product(layout=100) == -1
    for name in ("m", "n", "k"):
        assert product(**{name: -1}) == -4 and product(**{name: 1 << 31}) == -4
    assert product(m=1 << 30, n=1 << 30, ldc=1 << 30) == -4
    assert product(lda=299) == -5 and product(ldb=299) == -6
    assert product(ldc=5) == -7 and product(layout=COL, ldc=4) == -7
    for name in ("A", "B", "SA", "SB", "C"):
        assert product(**{name: None}) == -8
    assert product(C=None, alpha=0.0) == -8 and product(C=None, k=0) == -8
    assert product(c_type=3) == -20
    assert product(a_block=1) == -21 and product(b_block=1) == -21 and product(scales=0) == -21
    assert product(ldsa=2) == -23 and product(ldsb=2) == -23
    assert product(m=0, C=None) == 0 and product(n=0, A=None) == 0
    assert X.mg_block_gemm_workspace_bytes(-1, 2, 3) == 0 and X.mg_block_gemm_workspace_bytes(0, 2, 3) == 0


def test_grouped_product_refusals():
    def call(groups=3, offsets=FAKE, rows=9, n=6, k=300, A=FAKE, lda=300, SA=FAKE, ldsa=3, fan=2, b_block=X.MG_BLOCK_SQUARE, B=FAKE, ldb=300,
             stride_b=1800, SB=FAKE, ldsb=3, stride_sb=3, scales=X.MG_SCALES_POW2, c_type=X.MG_F32, C=FAKE, ldc=6, alpha=1.0):
        return X.mg_block_gemm_grouped(groups, offsets, rows, n, k, alpha, scales, A, lda, SA, ldsa, None, fan, b_block, B, ldb, stride_b, SB, ldsb, stride_sb, 0.0, c_type,
                                       C, ldc, None, 0, check=False)
    assert call(rows=-1) == -4 and call(n=-1) == -4 and call(k=-1) == -4
    assert call(lda=299) == -5 and call(ldb=299) == -6 and call(ldc=5) == -7
    for name in ("A", "B", "SA", "SB", "C", "offsets"):
        assert call(**{name: None}) == -8
    assert call(stride_b=-1) == -14 and call(stride_sb=-1) == -14
    assert call(c_type=7) == -20 and call(b_block=7) == -21 and call(scales=7) == -21
    assert call(groups=0) == -22 and call(groups=1025) == -22 and call(fan=0) == -22
    assert call(ldsa=2) == -23 and call(ldsb=2) == -23
    assert call(rows=0, offsets=None) == 0 and call(n=0, C=None) == 0
    assert X.mg_block_gemm_grouped_workspace_bytes(0, 5, 5, 5) == 0


def test_grouped_sum_refusals():
    def call(groups=3, offsets=FAKE, rows=100, m=5, n=6, A=FAKE, lda=512, SA=FAKE, ldsa=4, B=FAKE, ldb=512, SB=FAKE, ldsb=4, c_type=X.MG_F32, C=FAKE,
             ldc=6, stride_c=30, scales=X.MG_SCALES_POW2, alpha=1.0):
        return X.mg_block_gemm_grouped_sum(groups, offsets, rows, m, n, alpha, scales, A, lda, SA, ldsa, B, ldb, SB, ldsb, 0.0, c_type, C, ldc, stride_c, None, 0,
                                           check=False)
    assert call(rows=-1) == -4 and call(m=-1) == -4 and call(n=-1) == -4
    assert call(lda=511) == -5 and call(ldb=511) == -6 and call(ldc=5) == -7
    for name in ("A", "B", "SA", "SB", "C", "offsets"):
        assert call(**{name: None}) == -8
    assert call(stride_c=-1) == -14 and call(c_type=-2) == -20 and call(scales=0) == -21
    assert call(groups=0) == -22 and call(groups=2000) == -22
    assert call(ldsa=3) == -23 and call(ldsb=3) == -23
    assert call(m=0, C=None) == 0 and call(n=0, offsets=None) == 0
    assert X.mg_block_gemm_grouped_sum_workspace_bytes(0, 5, 5, 5) == 0


def test_routing_refusals():
    def sort(tokens=4, fan=2, experts=8, ids=FAKE, offsets=FAKE, position=FAKE, source=FAKE, ws=None):
        return X.mg_expert_sort(tokens, fan, experts, ids, offsets, position, source, ws, 0, check=False)
    assert sort(tokens=-1) == -4 and sort(tokens=1 << 30) == -4
    for name in ("ids", "offsets", "position", "source"):
        assert sort(**{name: None}) == -8
    assert sort(tokens=0, offsets=None) == -8
    assert sort(tokens=1 << 20) == -10
    assert sort(fan=0) == -22 and sort(fan=65) == -22 and sort(experts=0) == -22 and sort(experts=1025) == -22
    assert X.mg_expert_sort_workspace_bytes(8, 2, 8) == 0 and X.mg_expert_sort_workspace_bytes(1 << 20, 8, 64) > 0
    assert X.mg_expert_sort_workspace_bytes(-1, 2, 8) == 0 and X.mg_expert_sort_workspace_bytes(8, 0, 8) == 0

    def gather(dtype=X.MG_F32, tokens=4, fan=2, cols=10, A=FAKE, lda=10, index=FAKE, B=FAKE, ldb=10, fn=X.mg_expert_gather):
        return fn(dtype, tokens, fan, cols, A, lda, index, None, B, ldb, stream=0, check=False)
    for fn in (X.mg_expert_gather, X.mg_expert_combine):
        assert gather(fn=fn, tokens=-1) == -4 and gather(fn=fn, cols=-1) == -4 and gather(fn=fn, tokens=1 << 25) == -4
        assert gather(fn=fn, lda=9) == -5 and gather(fn=fn, ldb=9) == -6
        assert gather(fn=fn, A=None) == -8 and gather(fn=fn, index=None) == -8 and gather(fn=fn, B=None) == -8
        assert gather(fn=fn, dtype=5) == -20 and gather(fn=fn, fan=0) == -22
        assert gather(fn=fn, tokens=0, A=None) == 0 and gather(fn=fn, cols=0, B=None) == 0

    def grad(dtype=X.MG_F32, tokens=4, fan=2, cols=10, dO=FAKE, lddo=10, Y=FAKE, ldy=10, position=FAKE, dY=FAKE, lddy=10, dw=FAKE):
        return X.mg_expert_combine_grad(dtype, tokens, fan, cols, dO, lddo, Y, ldy, position, None, dY, lddy, dw, stream=0, check=False)
    assert grad(tokens=-1) == -4 and grad(lddo=9) == -5 and grad(ldy=9) == -6 and grad(lddy=9) == -7
    assert grad(dO=None) == -8 and grad(position=None) == -8 and grad(Y=None) == -8
    assert grad(dtype=5) == -20 and grad(fan=0) == -22 and grad(fan=65) == -22
    assert grad(dY=None, dw=None) == 0 and grad(tokens=0, dO=None) == 0


def test_wrong_types_raise():
    with pytest.raises(ctypes.ArgumentError):
        X.mg_expert_sort("tokens", 2, 8, None, None, None, None, None, 0)


def test_what_a_launch_holds():
    """Extents next to the limits: MG_ERR_NULL (-8) comes behind MG_ERR_DIM (-4) and shows that a size is taken."""
    last = (1 << 31) - 1025                       # an extent that kernels can still round up to whole blocks in 32 bits
    assert quantize(rows=1, cols=last, ldx=last, ldq=last, lds=1 << 24, X_=None) == -4           # (one row of that length: 2^24 blocks)
    assert quantize(rows=1, cols=1 << 27, ldx=1 << 27, ldq=1 << 27, lds=1 << 20, X_=None) == -8
    assert product(k=last, lda=last, ldb=last, C=None) == -8 and product(k=last + 1, lda=last + 1, ldb=last + 1, C=None) == -4

    def grouped(groups, rows, n):
        return X.mg_block_gemm_grouped(groups, FAKE, rows, n, 128, 1.0, X.MG_SCALES_POW2, FAKE, 128, FAKE, 1, None, 1, X.MG_BLOCK_SQUARE, FAKE, 128, 128 * n, FAKE, 1, n, 0.0,
                                       X.MG_BF16, None, n, None, 0, check=False)
    assert grouped(8, 16, 200000) == -8                                                          # few experts leave room for many columns
    assert grouped(1024, 16, 200000) == -4

    def rows(tokens, fan, cols, fn=X.mg_expert_combine):
        return fn(X.MG_F32, tokens, fan, cols, None, cols, FAKE, None, None, cols, stream=0, check=False)
    assert rows((1 << 24) - 1, 1, 4) == -8 and rows(1 << 24, 1, 4) == -4
    assert rows(1 << 20, 1, 8192) == -8 and rows(1 << 20, 1, 8193) == -4


def test_grouped_quantize_errors_in_order():
    def call(offsets, ldx):
        return X.mg_block_quantize_grouped(X.MG_F32, 2, offsets, 4, 8, FAKE, ldx, None, 1, FAKE, 8, FAKE, 1, None, 1, None, 1, stream=0, check=False)
    assert call(None, 7) == -5 and call(None, 8) == -8


def test_a_launch_of_2_to_32_threads_is_refused_as_a_size():
    """2^35 elements to quantise would be 2^24 work-groups of 256 threads, one more than a launch holds: a size (-4), not a launch that fails"""
    def call(rows, cols):
        tail = (None, cols, FAKE, cols, FAKE, cols >> 7, None, 1, None, 1)
        return X.mg_block_quantize(X.MG_BF16, X.MG_BLOCK_ROW, rows, cols, *tail, stream=0, check=False)
    assert call(1 << 18, 1 << 17) == -4 and call(1 << 21, 1 << 14) == -4
    assert call((1 << 18) - 128, 1 << 17) == -8 and call(1 << 18, (1 << 17) - 128) == -8

    def grouped(rows, groups, cols=1 << 14):
        return X.mg_block_quantize_grouped(X.MG_BF16, groups, FAKE, rows, cols, None, cols, None, 1, FAKE, cols, FAKE, cols >> 7, None, 1, None, 1, stream=0, check=False)
    assert grouped((1 << 21) - 128, 1) == -4 and grouped((1 << 21) - 256, 1) == -8

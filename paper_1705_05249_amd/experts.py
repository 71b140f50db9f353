"""Thin binding of include/mg_experts.h (8-bit products with a scale for each block of 128, routing of mixture-of-experts layers): same names
and argument order, in the manner of gemm.py.  A workspace argument stands for its address and its size.

Matrix arguments may be torch tensors on the GPU or raw integer device addresses; 8-bit matrices any tensor of one-byte elements
(torch.float8_e4m3fn among them).  The stream defaults to torch's current HIP stream.
"""
import ctypes

from . import gemm
from .gemm import MG_COL_MAJOR, MG_F16, MG_F32, MG_OK, MG_ROW_MAJOR, MgError  # noqa: F401  (callers take them from here)

MG_BF16 = 2
MG_BLOCK_ROW, MG_BLOCK_SQUARE = 151, 152
MG_SCALES_ANY, MG_SCALES_POW2 = 161, 162
MG_SUMS_FP32 = 1 << 16
MG_MOST_GROUPS, MG_MOST_FAN = 1024, 64
BLOCK = 128

_i, _l, _f, _p, _z = ctypes.c_int, ctypes.c_int64, ctypes.c_float, ctypes.c_void_p, ctypes.c_size_t
_result = [_p, _l, _p, _l]                        # an 8-bit matrix and its scales
_calls = {
    "mg_block_quantize": [_i, _i, _l, _l, _p, _l, *_result, *_result, _p],
    "mg_block_quantize_batched": [_i, _i, _l, _l, _l, _p, _l, _l, *[_p, _l, _l] * 4, _p],
    "mg_block_quantize_grouped": [_i, _i, _p, _l, _l, _p, _l, _p, _i, *_result, *_result, _p],
    "mg_block_gemm": [_i, _l, _l, _l, _f, _i, _i, *_result, _i, *_result, _f, _i, _p, _l, _p, _z, _p],
    "mg_block_gemm_grouped": [_i, _p, _l, _l, _l, _f, _i, *_result, _p, _i, _i, *[_p, _l, _l] * 2, _f, _i, _p, _l, _p, _z, _p],
    "mg_block_gemm_grouped_sum": [_i, _p, _l, _l, _l, _f, _i, *_result, *_result, _f, _i, _p, _l, _l, _p, _z, _p],
    "mg_expert_sort": [_l, _i, _i, _p, _p, _p, _p, _p, _z, _p],
    "mg_expert_gather": [_i, _l, _i, _l, _p, _l, _p, _p, _p, _l, _p],
    "mg_expert_combine": [_i, _l, _i, _l, _p, _l, _p, _p, _p, _l, _p],
    "mg_expert_combine_grad": [_i, _l, _i, _l, _p, _l, _p, _l, _p, _p, _p, _l, _p, _p],
}
_queries = {
    "mg_grouped_columns": ([_l, _i], _l),
    "mg_block_gemm_workspace_bytes": ([_l, _l, _l], _z),
    "mg_block_gemm_grouped_workspace_bytes": ([_i, _l, _l, _l], _z),
    "mg_block_gemm_grouped_sum_workspace_bytes": ([_i, _l, _l, _l], _z),
    "mg_expert_sort_workspace_bytes": ([_l, _i, _i], _z),
}
EXPORTS = (*_calls, *_queries)

_lib = None
_call = None


def lib():
    """the library of gemm.py with the types of these entry points"""
    global _lib
    if _lib is None:
        L = gemm.lib()
        for name, types in _calls.items():
            getattr(L, name).argtypes, getattr(L, name).restype = types, _i
        for name, (types, result) in _queries.items():
            getattr(L, name).argtypes, getattr(L, name).restype = types, result
        _lib = L
    return _lib


def _native():
    """the entry points with arguments taken as they are (csrc/python_call.cpp)"""
    global _call
    if _call is None:
        L, call = lib(), gemm._native()
        call.bind({name: ctypes.cast(getattr(L, name), _p).value for name in _calls}, gemm._stream_calls, gemm._by_ctypes)
        _call = call
    return _call


def _checked(status, name, check):
    if check and status != MG_OK:
        raise MgError(status, name)
    return status


def mg_block_quantize(dtype, block, rows, cols, X, ldx, Q, ldq, S, lds, T, ldt, ST, ldst, stream=None, check=True) -> int:
    st = (_call or _native()).mg_block_quantize(dtype, block, rows, cols, X, ldx, Q, ldq, S, lds, T, ldt, ST, ldst, stream)
    return _checked(st, "mg_block_quantize", check)


def mg_block_quantize_batched(dtype, block, batch, rows, cols, X, ldx, stride_x, Q, ldq, stride_q, S, lds, stride_s, T, ldt, stride_t, ST, ldst,
                              stride_st, stream=None, check=True) -> int:
    st = (_call or _native()).mg_block_quantize_batched(dtype, block, batch, rows, cols, X, ldx, stride_x, Q, ldq, stride_q, S, lds, stride_s,
                                                        T, ldt, stride_t, ST, ldst, stride_st, stream)
    return _checked(st, "mg_block_quantize_batched", check)


def mg_block_quantize_grouped(dtype, groups, offsets, rows, cols, X, ldx, source, fan, Q, ldq, S, lds, T, ldt, ST, ldst, stream=None,
                              check=True) -> int:
    st = (_call or _native()).mg_block_quantize_grouped(dtype, groups, offsets, rows, cols, X, ldx, source, fan, Q, ldq, S, lds, T, ldt, ST, ldst,
                                                        stream)
    return _checked(st, "mg_block_quantize_grouped", check)


def mg_grouped_columns(rows, groups) -> int:
    return lib().mg_grouped_columns(rows, groups)


def mg_block_gemm(layout, m, n, k, alpha, scales, a_block, A, lda, SA, ldsa, b_block, B, ldb, SB, ldsb, beta, c_type, C, ldc, workspace=None,
                  stream=None, check=True) -> int:
    st = (_call or _native()).mg_block_gemm(layout, m, n, k, alpha, scales, a_block, A, lda, SA, ldsa, b_block, B, ldb, SB, ldsb, beta, c_type, C,
                                            ldc, workspace, stream)
    return _checked(st, "mg_block_gemm", check)


def mg_block_gemm_workspace_bytes(m, n, k) -> int:
    return lib().mg_block_gemm_workspace_bytes(m, n, k)


def mg_block_gemm_grouped(groups, offsets, rows, n, k, alpha, scales, A, lda, SA, ldsa, source, fan, b_block, B, ldb, stride_b, SB, ldsb, stride_sb,
                          beta, c_type, C, ldc, workspace=None, stream=None, check=True) -> int:
    st = (_call or _native()).mg_block_gemm_grouped(groups, offsets, rows, n, k, alpha, scales, A, lda, SA, ldsa, source, fan, b_block, B, ldb,
                                                    stride_b, SB, ldsb, stride_sb, beta, c_type, C, ldc, workspace, stream)
    return _checked(st, "mg_block_gemm_grouped", check)


def mg_block_gemm_grouped_workspace_bytes(groups, rows, n, k) -> int:
    return lib().mg_block_gemm_grouped_workspace_bytes(groups, rows, n, k)


def mg_block_gemm_grouped_sum(groups, offsets, rows, m, n, alpha, scales, A, lda, SA, ldsa, B, ldb, SB, ldsb, beta, c_type, C, ldc, stride_c,
                              workspace=None, stream=None, check=True) -> int:
    st = (_call or _native()).mg_block_gemm_grouped_sum(groups, offsets, rows, m, n, alpha, scales, A, lda, SA, ldsa, B, ldb, SB, ldsb, beta, c_type,
                                                        C, ldc, stride_c, workspace, stream)
    return _checked(st, "mg_block_gemm_grouped_sum", check)


def mg_block_gemm_grouped_sum_workspace_bytes(groups, rows, m, n) -> int:
    return lib().mg_block_gemm_grouped_sum_workspace_bytes(groups, rows, m, n)


def mg_expert_sort(tokens, fan, experts, ids, offsets, position, source, workspace=None, stream=None, check=True) -> int:
    st = (_call or _native()).mg_expert_sort(tokens, fan, experts, ids, offsets, position, source, workspace, stream)
    return _checked(st, "mg_expert_sort", check)


def mg_expert_sort_workspace_bytes(tokens, fan, experts) -> int:
    return lib().mg_expert_sort_workspace_bytes(tokens, fan, experts)


def mg_expert_gather(dtype, tokens, fan, cols, X, ldx, source, weights, Y, ldy, stream=None, check=True) -> int:
    st = (_call or _native()).mg_expert_gather(dtype, tokens, fan, cols, X, ldx, source, weights, Y, ldy, stream)
    return _checked(st, "mg_expert_gather", check)


def mg_expert_combine(dtype, tokens, fan, cols, Y, ldy, position, weights, O, ldo, stream=None, check=True) -> int:  # noqa: E741
    st = (_call or _native()).mg_expert_combine(dtype, tokens, fan, cols, Y, ldy, position, weights, O, ldo, stream)
    return _checked(st, "mg_expert_combine", check)


def mg_expert_combine_grad(dtype, tokens, fan, cols, dO, lddo, Y, ldy, position, weights, dY, lddy, dweights, stream=None, check=True) -> int:
    st = (_call or _native()).mg_expert_combine_grad(dtype, tokens, fan, cols, dO, lddo, Y, ldy, position, weights, dY, lddy, dweights, stream)
    return _checked(st, "mg_expert_combine_grad", check)

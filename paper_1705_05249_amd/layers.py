"""Thin binding of include/mg_layers.h (gated feed-forward blocks, softmax cross entropy over a vocabulary, clipping of gradients): same names and
argument order, in the manner of gemm.py and experts.py.  A workspace argument, and `kept`, stands for its address and its size.

Matrix arguments may be torch tensors on the GPU or raw integer device addresses; the host arrays of the gradient calls torch tensors on the CPU
(int32 types, int64 addresses and sizes) or addresses of such arrays.  The stream defaults to torch's current HIP stream.
"""
import ctypes

from . import gemm
from .experts import MG_BF16
from .gemm import MG_F16, MG_F32, MG_OK, MgError  # noqa: F401  (callers take them from here)

MG_ACT_SILU, MG_ACT_GELU, MG_ACT_GELU_TANH, MG_ACT_RELU2 = 171, 172, 173, 174

_i, _l, _f, _p, _z = ctypes.c_int, ctypes.c_int64, ctypes.c_float, ctypes.c_void_p, ctypes.c_size_t
_matrix, _memory = [_p, _l], [_p, _z]
_calls = {
    "mg_gated_forward": [_i, _i, _l, _l, _l, *_matrix * 5, *_memory * 2, _p],
    "mg_gated_backward": [_i, _i, _l, _l, _l, *_matrix * 5, *_memory, *_matrix * 4, *_memory, _p],
    "mg_vocab_loss": [_i, _l, _l, _l, *_matrix * 2, _p, _p, _p, *_memory, _p],
    "mg_vocab_loss_grad": [_i, _l, _l, _l, *_matrix * 2, _p, _p, _p, *_matrix * 2, *_memory, _p],
    "mg_gradient_norm": [_l, _p, _p, _p, _p, *_memory, _p],
    "mg_gradient_clip": [_l, _p, _p, _p, _p, _f, _p, *_memory, _p],
}
_queries = {
    "mg_gated_forward_workspace_bytes": [_i, _l, _l, _l],
    "mg_gated_kept_bytes": [_i, _l, _l, _l],
    "mg_gated_backward_workspace_bytes": [_i, _l, _l, _l],
    "mg_vocab_loss_workspace_bytes": [_i, _l, _l, _l],
    "mg_vocab_loss_grad_workspace_bytes": [_i, _l, _l, _l],
    "mg_gradient_workspace_bytes": [_l],
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
        for name, types in _queries.items():
            getattr(L, name).argtypes, getattr(L, name).restype = types, _z
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


def mg_gated_forward(dtype, activation, tokens, width, hidden, X, ldx, WG, ldwg, WU, ldwu, WD, ldwd, Y, ldy, kept=None, workspace=None, stream=None, check=True) -> int:
    st = (_call or _native()).mg_gated_forward(dtype, activation, tokens, width, hidden, X, ldx, WG, ldwg, WU, ldwu, WD, ldwd, Y, ldy, kept, workspace, stream)
    return _checked(st, "mg_gated_forward", check)


def mg_gated_backward(dtype, activation, tokens, width, hidden, X, ldx, WG, ldwg, WU, ldwu, WD, ldwd, dY, lddy, kept, dX, lddx, dWG, lddwg, dWU, lddwu, dWD, lddwd,
                      workspace=None, stream=None, check=True) -> int:
    st = (_call or _native()).mg_gated_backward(dtype, activation, tokens, width, hidden, X, ldx, WG, ldwg, WU, ldwu, WD, ldwd, dY, lddy, kept, dX, lddx, dWG, lddwg, dWU, lddwu,
                                                dWD, lddwd, workspace, stream)
    return _checked(st, "mg_gated_backward", check)


def mg_vocab_loss(dtype, tokens, width, vocab, X, ldx, W, ldw, targets, loss, lse, workspace=None, stream=None, check=True) -> int:
    st = (_call or _native()).mg_vocab_loss(dtype, tokens, width, vocab, X, ldx, W, ldw, targets, loss, lse, workspace, stream)
    return _checked(st, "mg_vocab_loss", check)


def mg_vocab_loss_grad(dtype, tokens, width, vocab, X, ldx, W, ldw, targets, lse, weights, dX, lddx, dW, lddw, workspace=None, stream=None, check=True) -> int:
    st = (_call or _native()).mg_vocab_loss_grad(dtype, tokens, width, vocab, X, ldx, W, ldw, targets, lse, weights, dX, lddx, dW, lddw, workspace, stream)
    return _checked(st, "mg_vocab_loss_grad", check)


def mg_gradient_norm(count, types, sources, sizes, norm, workspace=None, stream=None, check=True) -> int:
    st = (_call or _native()).mg_gradient_norm(count, types, sources, sizes, norm, workspace, stream)
    return _checked(st, "mg_gradient_norm", check)


def mg_gradient_clip(count, types, sources, results, sizes, max_norm, norm, workspace=None, stream=None, check=True) -> int:
    st = (_call or _native()).mg_gradient_clip(count, types, sources, results, sizes, max_norm, norm, workspace, stream)
    return _checked(st, "mg_gradient_clip", check)


def mg_gated_forward_workspace_bytes(dtype, tokens, width, hidden) -> int:
    return lib().mg_gated_forward_workspace_bytes(dtype, tokens, width, hidden)


def mg_gated_kept_bytes(dtype, tokens, width, hidden) -> int:
    return lib().mg_gated_kept_bytes(dtype, tokens, width, hidden)


def mg_gated_backward_workspace_bytes(dtype, tokens, width, hidden) -> int:
    return lib().mg_gated_backward_workspace_bytes(dtype, tokens, width, hidden)


def mg_vocab_loss_workspace_bytes(dtype, tokens, width, vocab) -> int:
    return lib().mg_vocab_loss_workspace_bytes(dtype, tokens, width, vocab)


def mg_vocab_loss_grad_workspace_bytes(dtype, tokens, width, vocab) -> int:
    return lib().mg_vocab_loss_grad_workspace_bytes(dtype, tokens, width, vocab)


def mg_gradient_workspace_bytes(count) -> int:
    return lib().mg_gradient_workspace_bytes(count)

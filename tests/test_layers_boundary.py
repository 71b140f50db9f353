"""Host-side checks of include/mg_layers.h that need no GPU: symbols, every refusal, sizes, and that arguments arrive; what the layers of dense_layers.py refuse."""
import ctypes
import math
import os
import re
import subprocess
import sys

import pytest
import torch

from paper_1705_05249_amd import dense_layers as D, gemm as G, layers as L

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
FAKE = 0x10000         # never dereferenced: every call below fails validation or returns early
NULL, OK, DIM, LDA, LDB, LDC, WORKSPACE, TYPE, ACTIVATION, KEPT, LIMIT = -8, 0, -4, -5, -6, -7, -10, -20, -30, -31, -32


class Memory:
    """stands for device memory of a size"""

    def __init__(self, size, at=FAKE):
        self.size, self.at = size, at

    def data_ptr(self):
        return self.at

    def numel(self):
        return self.size

    def element_size(self):
        return 1


def test_header_symbols_are_exported():
    text = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "mg_layers.h")).read(), flags=re.S)
    assert sorted(set(re.findall(r"\b(mg_[a-z0-9_]+)\s*\(", text))) == sorted(L.EXPORTS)
    for name in L.EXPORTS:
        assert getattr(L.lib(), name) is not None
    assert all(G.status_string(code) != "unknown status" for code in (ACTIVATION, KEPT, LIMIT))


def test_every_argument_arrives():
    lib, call = L.lib(), L._native()
    try:
        for name in L._calls:
            types, seen, args, expected = getattr(lib, name).argtypes, [], [], []
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
            assert getattr(L, name)(*args, check=False) == -7          # the function of the module hands all of them on, in this order
            assert seen == expected, name
    finally:
        L._call = None
        L._native()


BIG = Memory(1 << 40)


def forward(dtype=L.MG_BF16, act=L.MG_ACT_SILU, tokens=3, width=10, hidden=7, X=FAKE, ldx=10, WG=FAKE, ldg=10, WU=FAKE, ldu=10, WD=FAKE, ldd=7, Y=FAKE, ldy=10, kept=None, ws=BIG):
    return L.mg_gated_forward(dtype, act, tokens, width, hidden, X, ldx, WG, ldg, WU, ldu, WD, ldd, Y, ldy, kept, ws, stream=0, check=False)


def test_forward_refusals():
    for name in ("tokens", "width", "hidden"):
        assert forward(**{name: -1}) == DIM and forward(**{name: 1 << 24}) == DIM
    assert forward(tokens=1 << 20, hidden=1 << 14, ldd=1 << 14) == DIM                                     # 2 hidden tokens results
    assert forward(ldx=9) == LDA and forward(ldx=1 << 40) == DIM
    assert forward(ldg=9) == LDB and forward(ldu=9) == LDB and forward(ldd=6) == LDB and forward(ldy=9) == LDC
    for name in ("X", "WG", "WU", "WD", "Y"):
        assert forward(**{name: None}) == NULL
    assert forward(ws=None) == WORKSPACE and forward(ws=Memory(8)) == WORKSPACE and forward(ws=Memory(1 << 30, FAKE + 128)) == WORKSPACE
    need = L.mg_gated_forward_workspace_bytes(L.MG_BF16, 3, 10, 7)
    assert need > 0 and forward(ws=Memory(need), act=0) == ACTIVATION and forward(ws=Memory(need - 1), act=0) == WORKSPACE
    assert forward(dtype=3) == TYPE and forward(act=170) == ACTIVATION and forward(act=175) == ACTIVATION
    kept = L.mg_gated_kept_bytes(L.MG_BF16, 3, 10, 7)
    assert kept > 0 and forward(kept=Memory(kept - 1)) == KEPT and forward(kept=Memory(kept, FAKE + 64)) == KEPT
    # no work: nothing is needed
    assert forward(tokens=0, X=None, Y=None, ws=None) == OK and forward(width=0, X=None, ldx=1, ws=None) == OK


def backward(dtype=L.MG_BF16, act=L.MG_ACT_SILU, tokens=3, width=10, hidden=7, X=FAKE, ldx=10, WG=FAKE, ldg=10, WU=FAKE, ldu=10, WD=FAKE, ldd=7, dY=FAKE, lddy=10, kept=BIG, dX=FAKE,
             lddx=10, dG=FAKE, lddg=10, dU=FAKE, lddu=10, dD=FAKE, lddd=7, ws=BIG):
    return L.mg_gated_backward(dtype, act, tokens, width, hidden, X, ldx, WG, ldg, WU, ldu, WD, ldd, dY, lddy, kept, dX, lddx, dG, lddg, dU, lddu, dD, lddd, ws, stream=0, check=False)


def test_backward_refusals():
    for name in ("tokens", "width", "hidden"):
        assert backward(**{name: -1}) == DIM and backward(**{name: 1 << 24}) == DIM
    assert backward(ldx=9) == LDA and backward(lddy=9) == LDA
    assert backward(ldg=9) == LDB and backward(ldu=9) == LDB and backward(ldd=6) == LDB
    assert backward(lddx=9) == LDC and backward(lddg=9) == LDC and backward(lddu=9) == LDC and backward(lddd=6) == LDC
    for name in ("X", "WG", "WU", "WD", "dY"):
        assert backward(**{name: None}) == NULL
    for name in ("dX", "dG", "dU", "dD"):
        assert backward(**{"ldd" + name[1].lower(): 0, name: None}, act=0) == ACTIVATION                   # a result that is not wanted needs no leading dimension
    assert backward(ws=None) == WORKSPACE
    need = L.mg_gated_backward_workspace_bytes(L.MG_BF16, 3, 10, 7)
    assert backward(ws=Memory(need), act=0) == ACTIVATION and backward(ws=Memory(need - 1), act=0) == WORKSPACE
    assert backward(dtype=-1) == TYPE and backward(kept=None) == KEPT and backward(kept=Memory(8)) == KEPT
    assert backward(dX=None, dG=None, dU=None, dD=None, X=None, ws=None, kept=None) == OK


def vocab(dtype=L.MG_F16, tokens=4, width=6, vocab=9, X=FAKE, ldx=6, W=FAKE, ldw=6, targets=FAKE, loss=FAKE, lse=FAKE, ws=BIG):
    return L.mg_vocab_loss(dtype, tokens, width, vocab, X, ldx, W, ldw, targets, loss, lse, ws, stream=0, check=False)


def vocab_grad(dtype=L.MG_F16, tokens=4, width=6, vocab=9, X=FAKE, ldx=6, W=FAKE, ldw=6, targets=FAKE, lse=FAKE, weights=None, dX=FAKE, lddx=6, dW=FAKE, lddw=6, ws=BIG):
    return L.mg_vocab_loss_grad(dtype, tokens, width, vocab, X, ldx, W, ldw, targets, lse, weights, dX, lddx, dW, lddw, ws, stream=0, check=False)


def test_loss_refusals():
    for fn in (vocab, vocab_grad):
        for name in ("tokens", "width", "vocab"):
            assert fn(**{name: -1}) == DIM and fn(**{name: 1 << 24}) == DIM
        assert fn(tokens=1 << 20, vocab=1 << 15) == DIM
        assert fn(ldx=5) == LDA and fn(ldw=5) == LDB and fn(ldw=1 << 38) == DIM
        for name in ("X", "W", "targets", "lse"):
            assert fn(**{name: None}) == NULL
        assert fn(ws=None) == WORKSPACE and fn(ws=Memory(16)) == WORKSPACE and fn(dtype=7) == TYPE
    assert vocab(loss=None) == NULL
    assert vocab_grad(lddx=5) == LDC and vocab_grad(lddw=5) == LDC
    assert vocab(tokens=0, X=None, targets=None, ws=None) == OK
    assert vocab_grad(dX=None, dW=None, X=None, targets=None, lse=None, ws=None) == OK


def clip(count=2, types=(0, 2), sources=(FAKE, FAKE), results=(FAKE, FAKE), sizes=(5, 9), max_norm=1.0, norm=FAKE, ws=BIG, fn="clip"):
    host = lambda v, kind=torch.int64: None if v is None else torch.tensor(v, dtype=kind)  # noqa: E731
    lists = host(types, torch.int32), host(sources), host(results), host(sizes)
    if fn == "norm":
        return L.mg_gradient_norm(count, lists[0], lists[1], lists[3], norm, ws, stream=0, check=False)
    return L.mg_gradient_clip(count, *lists, max_norm, norm, ws, stream=0, check=False)


def test_clip_refusals():
    for fn in ("clip", "norm"):
        assert clip(count=-1, fn=fn) == DIM and clip(count=(1 << 16) + 1, fn=fn) == DIM
        assert clip(sizes=(5, -1), fn=fn) == DIM and clip(sizes=(1 << 40, 1), fn=fn) == DIM
        for name in ("types", "sources", "sizes", "norm"):
            assert clip(**{name: None}, fn=fn) == NULL
        assert clip(sources=(FAKE, 0), fn=fn) == NULL
        assert clip(ws=None, fn=fn) == WORKSPACE and clip(ws=Memory(L.mg_gradient_workspace_bytes(2) - 1), fn=fn) == WORKSPACE
        assert clip(types=(0, 3), fn=fn) == TYPE and clip(types=(-1, 0), fn=fn) == TYPE
    assert clip(results=(0, FAKE)) == NULL
    assert clip(max_norm=-1.0) == LIMIT and clip(max_norm=math.nan) == LIMIT


def test_sizes_of_refused_and_empty_calls():
    for query in (L.mg_gated_forward_workspace_bytes, L.mg_gated_kept_bytes, L.mg_gated_backward_workspace_bytes, L.mg_vocab_loss_grad_workspace_bytes):
        assert query(3, 4, 4, 4) == 0 and query(0, -1, 4, 4) == 0 and query(0, 1 << 24, 4, 4) == 0 and query(0, 0, 4, 4) == 0 and query(0, 4, 4, 0) == 0
        assert all(query(code, 4, 4, 4) > 0 for code in (0, 1, 2))
    assert L.mg_vocab_loss_workspace_bytes(2, 0, 4, 4) == 0 and L.mg_vocab_loss_workspace_bytes(2, 4, 4, 4) > 0
    assert L.mg_gradient_workspace_bytes(0) == 0 and L.mg_gradient_workspace_bytes(-1) == 0 and L.mg_gradient_workspace_bytes(1) > 0 and L.mg_gradient_workspace_bytes((1 << 16) + 1) == 0


def test_layers_refuse_what_the_calls_would_believe():
    w, d = torch.zeros(6, 4), torch.zeros(4, 6)
    with pytest.raises(ValueError, match="expected hidden x width"):
        D.GatedBlock(w, w, w)
    with pytest.raises(ValueError, match="none of silu"):
        D.GatedBlock(w, w, d, "tanh")
    with pytest.raises(ValueError, match="the GPU"):
        D.GatedBlock(w, w, d)
    with pytest.raises(TypeError, match="float64"):
        D.GatedBlock(w.double(), w.double(), d.double())
    with pytest.raises(ValueError, match="expected vocab x width"):
        D.VocabLoss(torch.zeros(3))
    with pytest.raises(ValueError, match="the GPU"):
        D.VocabLoss(w)
    with pytest.raises(ValueError, match="the GPU"):
        D.Gradients([w])
    with pytest.raises(TypeError, match="int64"):
        D.Gradients([torch.zeros(3, dtype=torch.int64)])


def test_copies_of_matrices_without_columns():
    """width 0, with tokens from which copies of operands off 16 bytes start: nothing to copy.  In a process of its own, which sees no GPU: its launches fail"""
    program = """
import sys
from paper_1705_05249_amd import layers as L
for dtype in (L.MG_F16, L.MG_BF16, L.MG_F32):
    for tokens in (191, 192, 300, 5000):
        for ldx, ldw in ((1, 1), (8, 1), (1, 8), (8, 8), (3, 5)):
            st = L.mg_vocab_loss(dtype, tokens, 0, 7, None, ldx, None, ldw, 1 << 16, 1 << 16, 1 << 16, type("M", (), dict(data_ptr=lambda s: 1 << 16, numel=lambda s: 1 << 40, element_size=lambda s: 1))(), stream=0, check=False)
            assert st < 0, st
print("done")
"""
    run = subprocess.run([sys.executable, "-c", program], cwd=ROOT, env={**os.environ, "HIP_VISIBLE_DEVICES": "-1"}, capture_output=True, text=True)
    assert run.returncode == 0 and run.stdout.split()[-1] == "done", (run.returncode, run.stderr[-500:])


@pytest.mark.parametrize("dtype", [L.MG_F16, L.MG_BF16])
def test_the_gradient_of_the_loss_does_not_hold_a_slice_for_every_piece(dtype):
    """a copy of X, 2^28 elements of dz or 256 columns of them, copies of odd weights, four slices of dX and room for slices of a product: no tokens^2"""
    for tokens, width, vocab in ((8192, 2048, 65536), (32768, 4096, 131072), (65536, 4096, 131072), (131072, 4096, 131072), (131072, 8192, 131072), (1 << 20, 1024, 16000), (100001, 1001, 99999)):
        padded = -(-width // 64) * 64
        dz = 2 * max(1 << 28, tokens * (256 + 64))
        room = 64 << 20                                                   # 1024 tiles of 256 x 256 in FP32 are the most that slices of a product have
        most = (2 + 4 * 4) * tokens * padded + dz + 2 * 2 * vocab * padded * (width % 8 != 0) + 4 * room + 4096
        assert L.mg_vocab_loss_grad_workspace_bytes(dtype, tokens, width, vocab) <= most, (tokens, width, vocab)

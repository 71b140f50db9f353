"""Quantising in blocks of 128 against the definition in 64 bits: every byte and every scale has to be the same."""
import numpy as np
import pytest
import torch

from paper_1705_05249_amd import experts as X
from tests import expert_reference as R

pytestmark = pytest.mark.gpu
CODE = {"f32": X.MG_F32, "f16": X.MG_F16, "bf16": X.MG_BF16}
TYPE = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
FILL = 0xA5


def held(rows, cols, ld, start=0, kind=torch.uint8):
    """a buffer with `start` elements in front of a rows x ld matrix, filled with a pattern, and the matrix's first element's view"""
    buf = torch.full(((start + rows * ld + 64) * kind.itemsize,), FILL, dtype=torch.uint8, device="cuda").view(kind)
    return buf, buf[start:]


def matrix(buf, start, rows, cols, ld):
    return buf[start:start + rows * ld].view(rows, ld)[:, :cols].cpu().numpy()


def untouched(buf, start, rows, cols, ld):
    """everything but the rows x cols matrix still holds the pattern"""
    b = buf.view(torch.uint8).cpu().numpy().reshape(buf.numel(), -1).copy()
    b[start:start + rows * ld].reshape(rows, ld, -1)[:, :cols] = FILL
    return bool((b == FILL).all())


def inputs(rows, cols, kind, seed):
    rng = np.random.default_rng(seed)
    x = rng.standard_normal((rows, cols)) * np.exp(rng.standard_normal(cols))
    return torch.tensor(x).to(TYPE[kind])


def check(x, kind, square, sides, ldx, ldq, ldt, starts=(0, 0, 0)):
    rows, cols = x.shape
    xbuf = torch.zeros(starts[0] + rows * ldx + 8, dtype=TYPE[kind], device="cuda")
    xbuf[starts[0]:starts[0] + rows * ldx].view(rows, ldx)[:, :cols] = x.cuda()
    tall = -(-rows // 128) if square else rows
    wide = -(-cols // 128) if square else cols
    down, across = -(-rows // 128), -(-cols // 128)
    q, qv = held(rows, cols, ldq, starts[1])
    s, sv = held(tall, across, across + 1, 0, torch.float32)
    t, tv = held(cols, rows, ldt, starts[2])
    st, stv = held(wide, down, down + 2, 0, torch.float32)
    plain, turned = sides != "turned", sides != "plain"
    X.mg_block_quantize(CODE[kind], X.MG_BLOCK_SQUARE if square else X.MG_BLOCK_ROW, rows, cols, xbuf[starts[0]:], ldx,
                        qv if plain else None, ldq if plain else 0, sv if plain else None, across + 1 if plain else 0,
                        tv if turned else None, ldt if turned else 0, stv if turned else None, down + 2 if turned else 0)
    torch.cuda.synchronize()
    v = x.to(torch.float64).numpy()
    if plain:
        want, scales = R.quantize(v, square)
        assert np.array_equal(matrix(q, starts[1], rows, cols, ldq) & 0x7F == 0x7F, want & 0x7F == 0x7F)
        nan = want & 0x7F == 0x7F
        assert np.array_equal(np.where(nan, 0, matrix(q, starts[1], rows, cols, ldq)), np.where(nan, 0, want))
        assert np.array_equal(matrix(s, 0, tall, across, across + 1), scales.astype(np.float32))
        assert untouched(q, starts[1], rows, cols, ldq) and untouched(s, 0, tall, across, across + 1)
    if turned:
        want, scales = R.quantize(v.T, square)
        nan = want & 0x7F == 0x7F
        got = matrix(t, starts[2], cols, rows, ldt)
        assert np.array_equal(got & 0x7F == 0x7F, nan)
        assert np.array_equal(np.where(nan, 0, got), np.where(nan, 0, want))
        assert np.array_equal(matrix(st, 0, wide, down, down + 2), scales.astype(np.float32))
        assert untouched(t, starts[2], cols, rows, ldt) and untouched(st, 0, wide, down, down + 2)


SIZES = [(1, 1), (1, 128), (3, 129), (7, 1000), (16, 64), (127, 8), (128, 128), (129, 257), (300, 77), (1, 4096), (257, 384)]


@pytest.mark.parametrize("kind", ("f32", "f16", "bf16"))
@pytest.mark.parametrize("square", (False, True))
@pytest.mark.parametrize("sides", ("plain", "turned", "both"))
def test_sizes(kind, square, sides):
    for i, (rows, cols) in enumerate(SIZES):
        print(kind, square, sides, rows, cols, flush=True)
        check(inputs(rows, cols, kind, i), kind, square, sides, cols, cols, rows)


@pytest.mark.parametrize("kind", ("f32", "bf16"))
@pytest.mark.parametrize("starts", ((0, 0, 0), (1, 1, 1), (8, 16, 16), (3, 5, 7)))
def test_strides_and_alignment(kind, starts):
    for square in (False, True):
        check(inputs(130, 200, kind, 5), kind, square, "both", 203, 207, 131, starts)
        check(inputs(130, 208, kind, 6), kind, square, "both", 208, 208, 144, starts)


@pytest.mark.parametrize("square", (False, True))
def test_special_values(square):
    """zeros, signed zeros, infinities, NaN, the ends of the range, ties, and blocks whose maximum is at a scale's limit"""
    x = inputs(140, 300, "f32", 9).clone()
    x[0, :] = 0.0
    x[1, :128] = -0.0
    x[2, 5], x[3, 7], x[4, 130] = float("inf"), float("-inf"), float("nan")
    x[5, :128] = float("nan")
    x[6, 0] = 3.4028234663852886e38
    x[7, :] = 1e-45
    x[8, :] = 1.1754943508222875e-38
    x[9, :128] = torch.linspace(0, 448, 128)
    x[10, :128] = torch.arange(128) / 2.0
    x[11, 0], x[11, 1:128] = 448.0, 17.0 / 2 ** 7           # a tie between two steps
    x[12, 0] = 448.0 * (1 + 2.0 ** -23)
    x[13, 0] = 448.0 * 2.0 ** -20
    x[14, 128:256] = 2.0 ** -140
    check(x, "f32", square, "both", 300, 300, 140)
    h = x.clamp(-60000, 60000).to(torch.float16)
    check(h, "f16", square, "both", 300, 300, 140)


def test_every_e4m3_number_and_tie():
    """numbers of e4m3 and the points halfway between them, from a block that keeps its scale at one"""
    numbers = np.concatenate([R.E4M3[:0x7F], (R.E4M3[:0x7E] + R.E4M3[1:0x7F]) / 2])
    x = np.zeros((3, 128))
    x.reshape(-1)[:numbers.size] = numbers
    x[:, 127] = 448.0
    x = torch.tensor(np.concatenate([x, -x]), dtype=torch.float32)
    check(x, "f32", False, "plain", 128, 128, 6)


@pytest.mark.parametrize("square", (False, True))
def test_batched(square):
    batch, rows, cols = 3, 130, 150
    x = torch.stack([inputs(rows, cols, "bf16", 20 + b) for b in range(batch)])
    tall, wide = (2, 2) if square else (rows, cols)
    q, t = torch.zeros(batch, rows, 160, dtype=torch.uint8, device="cuda"), torch.zeros(batch, cols, 144, dtype=torch.uint8, device="cuda")
    s, st = torch.zeros(batch, tall, 2, device="cuda"), torch.zeros(batch, wide, 2, device="cuda")
    X.mg_block_quantize_batched(X.MG_BF16, X.MG_BLOCK_SQUARE if square else X.MG_BLOCK_ROW, batch, rows, cols, x.cuda(), cols, rows * cols,
                                q, 160, rows * 160, s, 2, tall * 2, t, 144, cols * 144, st, 2, wide * 2)
    torch.cuda.synchronize()
    for b in range(batch):
        v = x[b].to(torch.float64).numpy()
        for got, scales, have, width in ((q, s, v, cols), (t, st, v.T, rows)):
            want, ws = R.quantize(have, square)
            assert np.array_equal(got[b].cpu().numpy()[:, :width], want)
            assert np.array_equal(scales[b].cpu().numpy(), ws.astype(np.float32))


@pytest.mark.parametrize("counts,fan", (([5, 0, 130, 1, 0], 1), ([128, 256, 3], 2), ([0, 0, 1], 3), ([0, 0], 1), ([64] * 70 + [1], 2)))
def test_grouped(counts, fan):
    """rows of experts: gathered, each expert's transpose on blocks of its own with zeros to the block's end; rows of no expert untouched"""
    total, experts, cols = sum(counts), len(counts), 200
    rows = -(-(total + 3) // fan) * fan                      # some slots were dropped
    rng = np.random.default_rng(3)
    x = inputs(rows // fan, cols, "bf16", 11)
    source = np.full(rows, -1, np.int32)
    source[:total] = rng.permutation(rows)[:total]
    offsets = np.cumsum([0] + counts).astype(np.int32)
    columns = X.mg_grouped_columns(rows, experts)
    assert columns == -(-rows // 128) * 128 + 128 * experts
    q, qv = held(rows, cols, cols)
    s, sv = held(rows, 2, 2, 0, torch.float32)
    t, tv = held(cols, columns, columns)
    st, stv = held(cols, columns // 128, columns // 128, 0, torch.float32)
    X.mg_block_quantize_grouped(X.MG_BF16, experts, torch.tensor(offsets).cuda(), rows, cols, x.cuda(), cols, torch.tensor(source).cuda(), fan, qv, cols, sv, 2,
                                tv, columns, stv, columns // 128)
    torch.cuda.synchronize()
    v = x.to(torch.float64).numpy()[np.maximum(source, 0) // fan]
    want_q, want_s = np.full((rows, cols), FILL, np.uint8), matrix(s, 0, rows, 2, 2).copy()
    if total:
        want_q[:total], want_s[:total] = R.quantize(v[:total], False)
    assert np.array_equal(matrix(q, 0, rows, cols, cols), want_q)
    assert np.array_equal(matrix(s, 0, rows, 2, 2), want_s)
    pattern = np.frombuffer(bytes([FILL] * 4), np.float32)[0]
    assert (matrix(s, 0, rows, 2, 2)[total:] == pattern).all()
    want_t, want_st = np.full((cols, columns), FILL, np.uint8), np.full((cols, columns // 128), pattern, np.float32)
    for e in range(experts):
        lo, hi = offsets[e], offsets[e + 1]
        if lo == hi:
            continue
        at = R.group_column(int(lo), e)
        wide = -(-(hi - lo) // 128) * 128
        padded = np.zeros((cols, wide))
        padded[:, :hi - lo] = v[lo:hi].T
        want_t[:, at:at + wide], want_st[:, at // 128:(at + wide) // 128] = R.quantize(padded, False)
    assert np.array_equal(matrix(t, 0, cols, columns, columns), want_t)
    assert np.array_equal(matrix(st, 0, cols, columns // 128, columns // 128), want_st)


def test_offsets_past_32_bits():
    """a row that starts more than 2^32 elements behind the first"""
    ld = (1 << 31) + 4096
    x = torch.zeros(2 * ld + 128, dtype=torch.float16, device="cuda")
    x[2 * ld:] = torch.arange(128, device="cuda") / 8
    q = torch.zeros(2 * ld + 128, dtype=torch.uint8, device="cuda")
    s = torch.zeros(3, device="cuda")
    X.mg_block_quantize(X.MG_F16, X.MG_BLOCK_ROW, 3, 128, x, ld, q, ld, s, 1, None, 0, None, 0)
    torch.cuda.synchronize()
    want, scales = R.quantize((np.arange(128) / 8)[None], False)
    assert np.array_equal(q[2 * ld:].cpu().numpy(), want[0]) and float(s[2]) == scales[0, 0]


def test_another_stream():
    x, side = inputs(64, 256, "bf16", 1).cuda(), torch.cuda.Stream()
    q, s = torch.zeros(64, 256, dtype=torch.uint8, device="cuda"), torch.zeros(64, 2, device="cuda")
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        X.mg_block_quantize(X.MG_BF16, X.MG_BLOCK_ROW, 64, 256, x, 256, q, 256, s, 2, None, 0, None, 0)
    side.synchronize()
    want, scales = R.quantize(x.double().cpu().numpy(), False)
    assert np.array_equal(q.cpu().numpy(), want) and np.array_equal(s.cpu().numpy(), scales.astype(np.float32))

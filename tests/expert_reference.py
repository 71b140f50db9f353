"""The definitions of include/mg_experts.h in NumPy and 64 bits, element by element: what the GPU tests compare with."""
import numpy as np

BLOCK = 128


def _decode(byte):
    exponent, mantissa = (byte >> 3) & 15, byte & 7
    if exponent == 15 and mantissa == 7:
        value = np.nan
    elif exponent == 0:
        value = mantissa * 2.0 ** -9
    else:
        value = (8 + mantissa) * 2.0 ** (exponent - 10)
    return -value if byte & 128 else value


E4M3 = np.array([_decode(b) for b in range(256)])
_POSITIVE = E4M3[:0x7F]                                  # 0 .. 448, ascending


def round_e4m3(v):
    """bytes of the e4m3 numbers nearest to v (|v| <= 448), ties to the even mantissa"""
    a = np.abs(v)
    high = np.searchsorted(_POSITIVE, a).clip(0, 126)
    low = np.maximum(high - 1, 0)
    to_low, to_high = a - _POSITIVE[low], _POSITIVE[high] - a
    best = np.where((to_low < to_high) | ((to_low == to_high) & (low % 2 == 0)), low, high)
    return (best | np.where(np.signbit(v), 128, 0)).astype(np.uint8)


def scale_of(largest):
    """the smallest power of two, 2^-126 at least, with largest / scale <= 448; 1 for zeros"""
    e = -126
    if largest == 0:
        return 1.0
    while largest / 2.0 ** e > 448:
        e += 1
    return 2.0 ** e


def quantize(x, square):
    """(bytes, scales) of a float64 matrix"""
    rows, cols = x.shape
    tall = BLOCK if square else 1
    down, across = -(-rows // tall), -(-cols // BLOCK)
    q, s = np.zeros((rows, cols), np.uint8), np.ones((down, across))
    for i in range(down):
        for j in range(across):
            part = x[i * tall:(i + 1) * tall, j * BLOCK:(j + 1) * BLOCK]
            finite = np.isfinite(part)
            s[i, j] = scale_of(np.abs(part[finite]).max(initial=0.0))
            here = round_e4m3(np.where(finite, part, 0.0) / s[i, j])
            q[i * tall:(i + 1) * tall, j * BLOCK:(j + 1) * BLOCK] = np.where(finite, here, 0x7F)
    return q, s


def values(q, s, square):
    """what an 8-bit matrix stands for"""
    if square:
        s = np.repeat(s, BLOCK, 0)[:q.shape[0]]
    return E4M3[q] * np.repeat(s.astype(np.float64), BLOCK, 1)[:, :q.shape[1]]


def product(a, b, alpha=1.0, beta=0.0, c=None):
    """(result, sum of magnitudes) of alpha * a b^T + beta * c on values"""
    r, d = alpha * (a @ b.T), abs(alpha) * (np.abs(a) @ np.abs(b).T)
    if beta:
        r, d = r + beta * c, d + abs(beta) * np.abs(c)
    return r, d


#: unit roundoff and half of the smallest step of the element types
ROUNDOFF = {"f32": (2.0 ** -24, 0.0), "f16": (2.0 ** -11, 2.0 ** -25), "bf16": (2.0 ** -8, 0.0)}


def product_bound(result, magnitudes, k, kind):
    """How far a product may be off.  Products of two e4m3 numbers are exact in FP32; a matrix instruction adds up to 128 of them, blocks are scaled
    (two roundings) and added, slices and alpha, beta * C add eight more at most: 128 + 3 * blocks + 8 operations, each off by 2^-23 of
    the sum of magnitudes if it truncates; and the result's rounding."""
    unit, least = ROUNDOFF[kind]
    steps = min(k, BLOCK) + 3 * -(-k // BLOCK) + 8
    accumulated = steps * 2.0 ** -23 * magnitudes
    return accumulated + unit * (np.abs(result) + accumulated) + least


def near(got, want, bound, kind):
    """got is within `bound` of want; what lies beyond FP16's largest number (65504, half a step of 32 above it) has become infinite"""
    limit = 65520.0 if kind == "f16" else np.inf
    infinite = np.isinf(got) & (np.sign(got) == np.sign(want)) & (np.abs(want) + bound >= limit)
    finite = np.abs(want) - bound < limit
    return bool((infinite | (finite & (np.abs(got - want) <= bound))).all())


def sort(ids, experts):
    """(offsets, position, source) of flat slots, by insertion"""
    lists = [[i for i, e in enumerate(ids) if e == x] for x in range(experts)]
    order = [i for part in lists for i in part]
    offsets = np.cumsum([0] + [len(part) for part in lists])
    position, source = np.full(len(ids), -1), np.full(len(ids), -1)
    for row, slot in enumerate(order):
        position[slot], source[row] = row, slot
    return offsets.astype(np.int32), position.astype(np.int32), source.astype(np.int32)


def group_column(start, group):
    return -(-start // BLOCK) * BLOCK + BLOCK * group

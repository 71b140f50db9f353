"""The operators of mg_layers.h in 64 bits, each with a bound of what a kernel may be off, element by element.

The bounds follow the roundings of the formulas: a sum of k products of exact operands in FP32 is off by at most k steps of 2^-23 of the sum of
magnitudes (a step and not half of one, for matrix pipes that do not round to nearest); the exponential of x by at most 2^-23 (1 + |x|) of itself; a
number that is rounded to a type by half a step, eps / 2 of itself, or half the smallest number of FP16; errors of operands go through the
products as they stand.
"""
import math

import torch

HALF = {torch.float32: 2.0 ** -24, torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}     # half a step, of a number's magnitude
TINY = {torch.float32: 0.0, torch.float16: 2.0 ** -25, torch.bfloat16: 0.0}
STEP = 2.0 ** -23
ACTS = ("silu", "gelu", "gelu_tanh", "relu2")


def act(g, kind):
    """(act(g), its slope, the magnitude of what is exponentiated on the way)"""
    if kind == "silu":
        p = torch.sigmoid(g)
        return g * p, p * (1 + g * (1 - p)), g.abs()
    if kind == "relu2":
        v = g.clamp(min=0)
        return v * v, 2 * v, torch.zeros_like(g)
    if kind == "gelu":
        below = torch.special.ndtr(g)
        return g * below, below + g * torch.exp(-0.5 * g * g) / math.sqrt(2 * math.pi), g * g
    a, b = math.sqrt(2 / math.pi), 0.044715
    p = torch.sigmoid(2 * a * (g + b * g ** 3))
    return g * p, p + g * p * (1 - p) * 2 * a * (1 + 3 * b * g * g), (2 * a * (g + b * g ** 3)).abs()


def rounded(value, error, dtype):
    """bound of what was off by `error` and has been rounded"""
    return error + HALF[dtype] * (value.abs() + error) + TINY[dtype]


def product(a, ea, b, eb):
    """a @ b and its bound, for operands that are off by ea and eb (zero: exact)"""
    k = a.shape[1]
    size = (a.abs() + ea) @ (b.abs() + eb)
    return a @ b, ea @ b.abs() + a.abs() @ eb + ea @ eb + (k + 1) * STEP * size


def zero(x):
    return torch.zeros_like(x)


def block(x, wg, wu, wd, kind, dtype, dy=None):
    """{name: (value, bound)} of Y and, with dy, of the four gradients"""
    x, wg, wu, wd = (t.double() for t in (x, wg, wu, wd))
    g, eg = product(x, zero(x), wg.T, zero(wg.T))
    u, eu = product(x, zero(x), wu.T, zero(wu.T))
    a, slope, size = act(g, kind)
    curve = 2.0                                                   # no activation's second derivative is larger
    fine = 2.0 ** -22 * (4 + size)
    ea = slope.abs() * eg + curve * eg * eg + fine * a.abs()
    h = a * u
    eh = rounded(h, ea * u.abs() + (a.abs() + ea) * eu + 2 * STEP * h.abs(), dtype)
    y, ey = product(h, eh, wd.T, zero(wd.T))
    out = {"y": (y, rounded(y, ey, dtype))}
    if dy is None:
        return out
    dy = dy.double()
    dh, edh = product(dy, zero(dy), wd, zero(wd))
    es = curve * eg + fine * (1 + g.abs()) * (slope.abs() + 0.1)
    b = u * slope
    eb = eu * slope.abs() + (u.abs() + eu) * es + 2 * STEP * b.abs()
    if dtype == torch.bfloat16:                                   # kept with 11 bits, and an exponent for four
        ea, eb = (e + 2.0 ** -11 * (v.abs() + e) + 2.0 ** -38 * (v.abs() + e).amax() for v, e in ((a, ea), (b, eb)))
    dg, du = dh * b, dh * a
    edg = edh * b.abs() + (dh.abs() + edh) * eb + 3 * STEP * dg.abs()
    edu = edh * a.abs() + (dh.abs() + edh) * ea + 3 * STEP * du.abs()
    edg, edu = rounded(dg, edg, dtype), rounded(du, edu, dtype)
    d, ed = torch.cat((dg, du), 1), torch.cat((edg, edu), 1)
    w = torch.cat((wg, wu))
    hidden = wg.shape[0]
    dx = product(d, ed, w, zero(w))
    dw = product(d.T, ed.T, x, zero(x))
    dwd = product(dy.T, zero(dy.T), h, eh)
    # (one more rounding to FP32 between the two halves of dX, of half a step)
    out["dx"] = (dx[0], rounded(dx[0], dx[1] + STEP * dx[0].abs(), dtype))
    out["dwg"] = tuple(t[:hidden] for t in (dw[0], rounded(*dw, dtype)))
    out["dwu"] = tuple(t[hidden:] for t in (dw[0], rounded(*dw, dtype)))
    out["dwd"] = (dwd[0], rounded(*dwd, dtype))
    return out


def loss(x, w, targets, dtype, weights=None, gradient=False):
    """{name: (value, bound)} of loss and lse and, with gradient, of dx and dw"""
    x, w = x.double(), w.double()
    vocab = w.shape[0]
    z, ez = product(x, zero(x), w.T, zero(w.T))
    lse = torch.logsumexp(z, 1)
    counts = (targets >= 0) & (targets < vocab)
    at = torch.where(counts, targets, 0)
    far = (z - lse[:, None]).abs()
    # a sum of exponentials: each off by 2^-23 (1 + its exponent) and its share of the sum; additions: a tile's columns one by one in a lane, lanes and
    # tiles joined with two more exponentials each
    tiles = -(-vocab // 64)
    p = torch.exp(z - lse[:, None])
    elog = (p * (ez + 2 * STEP * (2 + far))).sum(1) + STEP * (40 + 2 * min(tiles, 16 + tiles // 16))
    elog = elog + elog ** 2 + STEP * lse.abs()
    picked = z.gather(1, at[:, None])[:, 0] if vocab else lse
    epicked = ez.gather(1, at[:, None])[:, 0] if vocab else elog
    value = torch.where(counts, lse - picked, 0.0)
    out = {"lse": (lse, elog), "loss": (value, torch.where(counts, elog + epicked + STEP * (lse.abs() + value.abs()), 0.0))}
    if not gradient:
        return out
    weights = torch.ones_like(lse) if weights is None else weights.double()
    wt = torch.where(counts, weights, 0.0)[:, None]
    here = torch.zeros_like(z)
    here[torch.arange(len(targets), device=z.device), at] = 1.0
    dz = wt * (p - here)
    # (the lse that the gradient is given was rounded to FP32 and is off as above)
    ep = p * (ez + elog[:, None] + STEP * (3 + far)) * 1.01 + 2 * STEP * (p + here)
    edz = wt.abs() * ep + 4 * STEP * dz.abs()
    largest = weights.abs().max()
    edz = edz + HALF[dtype] * (dz.abs() + edz) + TINY[dtype] * largest * 2.0 ** -13 * (wt != 0)
    dx, dw = product(dz, edz, w, zero(w)), product(dz.T, edz.T, x, zero(x))
    pieces = 2 * STEP * (1 + vocab // 256)                         # pieces of the vocabulary are added in FP32
    out["dx"] = (dx[0], rounded(dx[0], dx[1] + pieces * (dz.abs() @ w.abs()), dtype))
    out["dw"] = (dw[0], rounded(*dw, dtype))
    return out


def check(got, want, name):
    """got (on any device) is within its bound"""
    value, bound = want
    got = got.to(value.device).double()
    assert got.shape == value.shape, (name, got.shape, value.shape)
    if not got.numel():
        return
    off = (got - value).abs()
    bad = ~(off <= bound)
    assert not bool(bad.any()), (name, int(bad.sum()), float((off / bound.clamp(min=1e-300)).nan_to_num(nan=math.inf).max()), bad.nonzero()[:4].tolist())

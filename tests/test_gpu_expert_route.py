"""Sorting by expert, gathering, combining and the gradient of that, against plain loops in 64 bits and against differences."""
import numpy as np
import pytest
import torch

from paper_1705_05249_amd import experts as X
from tests import expert_reference as R

pytestmark = pytest.mark.gpu
CODE = {"f32": X.MG_F32, "f16": X.MG_F16, "bf16": X.MG_BF16}
TYPE = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}


def sorted_on_gpu(ids, tokens, fan, experts):
    slots = tokens * fan
    given = torch.tensor(ids, dtype=torch.int32).cuda()
    out = [torch.full((count + 4,), -77, dtype=torch.int32, device="cuda") for count in (experts + 1, slots, slots)]
    need = X.mg_expert_sort_workspace_bytes(tokens, fan, experts)
    ws = torch.empty(need, dtype=torch.uint8, device="cuda") if need else None
    X.mg_expert_sort(tokens, fan, experts, given, *out, ws)
    torch.cuda.synchronize()
    for x, count in zip(out, (experts + 1, slots, slots)):
        assert (x[count:] == -77).all(), "written behind an array"
    return [x[:count].cpu().numpy() for x, count in zip(out, (experts + 1, slots, slots))]


@pytest.mark.parametrize("tokens,fan,experts", ((0, 2, 5), (1, 1, 1), (1, 8, 8), (7, 2, 3), (64, 1, 64), (65, 3, 17), (1000, 2, 256), (4096, 2, 33), (4097, 2, 8),
                                                (5000, 7, 1024), (20011, 3, 300), (1 << 17, 1, 5)))
def test_sort(tokens, fan, experts):
    rng = np.random.default_rng(tokens)
    for kind in ("any", "one", "dropped", "none"):
        print(tokens, fan, experts, kind, flush=True)
        ids = rng.integers(0, experts, tokens * fan)
        if kind == "one":
            ids[:] = experts - 1
        if kind == "dropped":
            ids[rng.random(ids.size) < 0.3] = rng.choice([-1, experts, 1 << 30, -(1 << 31)])
        if kind == "none":
            ids[:] = -1
        got = sorted_on_gpu(ids, tokens, fan, experts)
        key = np.where((ids >= 0) & (ids < experts), ids, experts)
        order = np.argsort(key, kind="stable")
        offsets = np.concatenate([[0], np.cumsum(np.bincount(key, minlength=experts + 1)[:experts])]) if ids.size else np.zeros(experts + 1)
        total = int(offsets[-1])
        position, source = np.full(ids.size, -1), np.full(ids.size, -1)
        position[order[:total]], source[:total] = np.arange(total), order[:total]
        for name, x, y in zip(("offsets", "position", "source"), got, (offsets, position, source)):
            assert np.array_equal(x, y), (kind, name)
        if ids.size <= 200:
            assert all(np.array_equal(x, y) for x, y in zip(got, R.sort(ids.tolist(), experts)))


@pytest.mark.parametrize("slots,experts", ((64 * 4096, 7), (64 * 4096 + 1, 65), (1 << 20, 1024), ((1 << 21) + 4095, 3)))
def test_sort_of_many(slots, experts):
    rng = np.random.default_rng(slots)
    ids = rng.integers(-1, experts + 1, slots)
    ids[: slots // 3] = experts // 2                                       # one expert has most of the first chunks
    offsets, position, source = sorted_on_gpu(ids, slots, 1, experts)
    key = np.where((ids >= 0) & (ids < experts), ids, experts)
    order = np.argsort(key, kind="stable")
    want = np.concatenate([[0], np.cumsum(np.bincount(key, minlength=experts + 1)[:experts])])
    total = int(want[-1])
    where = np.full(slots, -1)
    where[order[:total]] = np.arange(total)
    assert np.array_equal(offsets, want) and np.array_equal(position, where)
    assert np.array_equal(source, np.where(np.arange(slots) < total, order, -1))


def routes(rng, tokens, fan, experts, dropped):
    ids = rng.integers(0, experts, tokens * fan)
    ids[rng.random(ids.size) < dropped] = -1
    return R.sort(ids.tolist(), experts)


CASES = [(1, 1, 1, 1), (3, 2, 4, 7), (5, 3, 2, 130), (40, 8, 16, 64), (33, 2, 5, 2051), (200, 4, 9, 96)]


@pytest.mark.parametrize("kind", ("f32", "f16", "bf16"))
@pytest.mark.parametrize("dropped", (0.0, 0.4))
@pytest.mark.parametrize("pad", (0, 5))
def test_gather_and_combine(kind, dropped, pad):
    unit, least = R.ROUNDOFF[kind]
    for tokens, fan, experts, cols in CASES:
        print(kind, dropped, pad, tokens, fan, experts, cols, flush=True)
        rng = np.random.default_rng(cols)
        offsets, position, source = routes(rng, tokens, fan, experts, dropped)
        slots, total = tokens * fan, offsets[-1]
        x = torch.tensor(rng.standard_normal((tokens, cols + pad))).to(TYPE[kind])
        w = torch.tensor(rng.uniform(-1, 1, slots), dtype=torch.float32)
        xv, wv = x.double().numpy()[:, :cols], w.double().numpy()
        for weights in (None, w.cuda()):
            y = torch.full((slots, cols + pad), 9.0, dtype=TYPE[kind], device="cuda")
            X.mg_expert_gather(CODE[kind], tokens, fan, cols, x.cuda(), cols + pad, torch.tensor(source).cuda(), weights, y, cols + pad)
            torch.cuda.synchronize()
            want = np.zeros((slots, cols))
            want[:total] = xv[source[:total] // fan] * (wv[source[:total]][:, None] if weights is not None else 1)
            got = y.double().cpu().numpy()
            assert (np.abs(got[:, :cols] - want) <= (unit + 2.0 ** -23) * np.abs(want) + least).all() and (got[:, cols:] == 9.0).all()
            if weights is None:
                assert np.array_equal(got[:, :cols], want)
        rows = torch.tensor(rng.standard_normal((slots, cols + pad))).to(TYPE[kind])
        rows[total:] = float("nan")                                       # rows of no slot do not count
        rv = rows.double().numpy()[:, :cols]
        for weights in (None, w.cuda()):
            o = torch.full((tokens, cols + pad), 9.0, dtype=TYPE[kind], device="cuda")
            X.mg_expert_combine(CODE[kind], tokens, fan, cols, rows.cuda(), cols + pad, torch.tensor(position).cuda(), weights, o, cols + pad)
            torch.cuda.synchronize()
            want, size = np.zeros((tokens, cols)), np.zeros((tokens, cols))
            for s, row in enumerate(position):
                if row >= 0:
                    term = rv[row] * (wv[s] if weights is not None else 1)
                    want[s // fan] += term
                    size[s // fan] += np.abs(term)
            got = o.double().cpu().numpy()
            bound = unit * np.abs(want) + (fan + 1) * 2.0 ** -23 * size + least          # a rounding for each addition, one at the end
            assert (np.abs(got[:, :cols] - want) <= bound).all() and (got[:, cols:] == 9.0).all()


@pytest.mark.parametrize("kind", ("f32", "f16", "bf16"))
@pytest.mark.parametrize("dropped", (0.0, 0.4, 1.0))
@pytest.mark.parametrize("pad", (0, 3))
def test_combine_gradient(kind, dropped, pad):
    unit, least = R.ROUNDOFF[kind]
    for tokens, fan, experts, cols in CASES + [(6, 2, 3, 9000)]:
        print(kind, dropped, pad, tokens, fan, experts, cols, flush=True)
        rng = np.random.default_rng(cols + 1)
        offsets, position, source = routes(rng, tokens, fan, experts, dropped)
        slots, total, ld = tokens * fan, offsets[-1], cols + pad
        g, y = (torch.tensor(rng.standard_normal((r, ld))).to(TYPE[kind]) for r in (tokens, slots))
        y[total:] = float("nan")
        w = torch.tensor(rng.uniform(-1, 1, slots), dtype=torch.float32)
        gv, yv, wv = g.double().numpy()[:, :cols], y.double().numpy()[:, :cols], w.double().numpy()
        at = torch.tensor(position).cuda()
        dy, dw = torch.full((slots, ld), 9.0, dtype=TYPE[kind], device="cuda"), torch.full((slots + 4,), 9.0, device="cuda")
        X.mg_expert_combine_grad(CODE[kind], tokens, fan, cols, g.cuda(), ld, y.cuda(), ld, at, w.cuda(), dy, ld, dw)
        torch.cuda.synchronize()
        got_y, got_w = dy.double().cpu().numpy(), dw.double().cpu().numpy()
        assert (got_y[total:] == 9.0).all() and (got_y[:, cols:] == 9.0).all() and (got_w[slots:] == 9.0).all()
        for s, row in enumerate(position):
            if row < 0:
                assert got_w[s] == 0.0
                continue
            want = wv[s] * gv[s // fan]
            assert (np.abs(got_y[row, :cols] - want) <= (unit + 2.0 ** -23) * np.abs(want) + least).all()
            terms = gv[s // fan] * yv[row]
            assert abs(got_w[s] - terms.sum()) <= (cols + 8) * 2.0 ** -24 * np.abs(terms).sum()
        # either result alone is the same result
        alone_y, alone_w = torch.full_like(dy, 9.0), torch.full_like(dw, 9.0)
        X.mg_expert_combine_grad(CODE[kind], tokens, fan, cols, g.cuda(), ld, None, 0, at, w.cuda(), alone_y, ld, None)
        X.mg_expert_combine_grad(CODE[kind], tokens, fan, cols, g.cuda(), ld, y.cuda(), ld, at, None, None, 0, alone_w)
        torch.cuda.synchronize()
        assert torch.equal(alone_y, dy) and torch.equal(alone_w, dw)


def test_gradient_against_differences():
    """FP32: the loss sum(O * G) changes by what the gradients say when Y or the weights change"""
    tokens, fan, experts, cols = 6, 2, 3, 40
    rng = np.random.default_rng(8)
    _, position, _ = routes(rng, tokens, fan, experts, 0.2)
    slots, at = tokens * fan, torch.tensor(position).cuda()
    y, g = (torch.tensor(rng.standard_normal((r, cols)), dtype=torch.float32).cuda() for r in (slots, tokens))
    w = torch.tensor(rng.uniform(0.2, 1, slots), dtype=torch.float32).cuda()

    def loss(y, w):
        o = torch.empty(tokens, cols, device="cuda")
        X.mg_expert_combine(X.MG_F32, tokens, fan, cols, y, cols, at, w, o, cols)
        return float((o.double() * g.double()).sum())
    dy, dw = torch.zeros_like(y), torch.zeros_like(w)
    X.mg_expert_combine_grad(X.MG_F32, tokens, fan, cols, g, cols, y, cols, at, w, dy, cols, dw)
    step = 2.0 ** -6
    for i in rng.integers(0, slots * cols, 10):
        up, down = y.clone(), y.clone()
        up.view(-1)[i] += step
        down.view(-1)[i] -= step
        # linear in y: only FP32 roundings of outputs around 2 separate the two, 2^-22 each over 2 * 2^-6
        assert abs((loss(up, w) - loss(down, w)) / (2 * step) - float(dy.view(-1)[i])) <= 2.0 ** -14
    for s in range(slots):
        up, down = w.clone(), w.clone()
        up[s] += step
        down[s] -= step
        assert abs((loss(y, up) - loss(y, down)) / (2 * step) - float(dw[s])) <= 40 * 2.0 ** -14


def test_combine_is_the_gradient_of_gather():
    """<gather(x), r> = <x, combine(r)> for whole numbers, exactly"""
    tokens, fan, experts, cols = 50, 3, 7, 100
    rng = np.random.default_rng(1)
    _, position, source = routes(rng, tokens, fan, experts, 0.3)
    x, r = (torch.tensor(rng.integers(-4, 5, (n, cols)), dtype=torch.float32).cuda() for n in (tokens, tokens * fan))
    y, o = torch.empty(tokens * fan, cols, device="cuda"), torch.empty(tokens, cols, device="cuda")
    X.mg_expert_gather(X.MG_F32, tokens, fan, cols, x, cols, torch.tensor(source).cuda(), None, y, cols)
    X.mg_expert_combine(X.MG_F32, tokens, fan, cols, r, cols, torch.tensor(position).cuda(), None, o, cols)
    torch.cuda.synchronize()
    assert float((y.double() * r.double()).sum()) == float((x.double() * o.double()).sum())


def test_offsets_past_32_bits():
    """a row more than 2^32 elements behind the first, in every matrix"""
    ld = (1 << 31) + 64
    x = torch.zeros(2 * ld + 64, dtype=torch.bfloat16, device="cuda")
    x[2 * ld:] = 3.0
    source = torch.tensor([2, 0, 1], dtype=torch.int32).cuda()
    y = torch.zeros(2 * ld + 64, dtype=torch.bfloat16, device="cuda")
    X.mg_expert_gather(X.MG_BF16, 3, 1, 64, x, ld, source, None, y, ld)
    torch.cuda.synchronize()
    assert (y[:64] == 3.0).all() and (y[2 * ld:] == 0.0).all()
    position = torch.tensor([1, 0, 2], dtype=torch.int32).cuda()
    X.mg_expert_combine(X.MG_BF16, 3, 1, 64, x, ld, position, None, y, ld)
    torch.cuda.synchronize()
    assert (y[2 * ld:] == 3.0).all() and (y[:64] == 0.0).all()
    dw = torch.zeros(3, device="cuda")
    X.mg_expert_combine_grad(X.MG_BF16, 3, 1, 64, x, ld, x, ld, position, None, y, ld, dw)
    torch.cuda.synchronize()
    assert dw.tolist() == [0.0, 0.0, 9.0 * 64]

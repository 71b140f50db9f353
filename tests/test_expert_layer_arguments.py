"""What expert_layer.py does with its arguments, without a GPU: tensors without memory, calls that are recorded instead of made.  No call may address
more memory than the tensors behind it hold, whatever the types and shapes that a program hands over."""
import inspect

import pytest
import torch
from torch._subclasses.fake_tensor import FakeTensorMode

from paper_1705_05249_amd import experts as X
from paper_1705_05249_amd import expert_layer as L
from paper_1705_05249_amd.expert_layer import INDEX_TYPES

BYTES = {X.MG_F32: 4, X.MG_F16: 2, X.MG_BF16: 2}
TOKENS, WIDTH, HIDDEN, EXPERTS, FAN = 64, 128, 160, 5, 2


def blocks(size):
    return -(-size // 128)


def holds(name, tensor, elements, size):
    if tensor is None or elements <= 0:
        return
    assert tensor.is_cuda, name
    held = tensor.untyped_storage().nbytes() - tensor.storage_offset() * tensor.element_size()
    assert elements * size <= held, f"{name}: {elements * size} bytes addressed, {held} held"


def matrix(name, tensor, rows, cols, ld, size):
    holds(name, tensor, (rows - 1) * ld + cols if rows > 0 and cols > 0 else 0, size)


def result(a, names, rows, cols, square=False, each=1):
    """an 8-bit matrix and its scales; of `each` experts"""
    (q, s), (ldq, lds) = names[:2], (a[names[2]], a[names[3]])
    tall = blocks(rows) if square else rows
    step_q, step_s = (a[names[4]], a[names[5]]) if each > 1 else (0, 0)
    holds(q, a[q], (each - 1) * step_q + (rows - 1) * ldq + cols, 1)
    holds(s, a[s], (each - 1) * step_s + (tall - 1) * lds + blocks(cols), 4)


def quantize(a):
    matrix("X", a["X"], a["rows"], a["cols"], a["ldx"], BYTES[a["dtype"]])
    if a["Q"] is not None:
        result(a, ("Q", "S", "ldq", "lds"), a["rows"], a["cols"])
    if a["T"] is not None:
        result(a, ("T", "ST", "ldt", "ldst"), a["cols"], a["rows"])


def quantize_batched(a):
    z, rows, cols, batch = BYTES[a["dtype"]], a["rows"], a["cols"], a["batch"]
    holds("X", a["X"], (batch - 1) * a["stride_x"] + (rows - 1) * a["ldx"] + cols, z)
    result(a, ("Q", "S", "ldq", "lds", "stride_q", "stride_s"), rows, cols, True, batch)
    result(a, ("T", "ST", "ldt", "ldst", "stride_t", "stride_st"), cols, rows, True, batch)


def quantize_grouped(a):
    rows, cols = a["rows"], a["cols"]
    matrix("X", a["X"], -(-rows // a["fan"]) if a["source"] is not None else rows, cols, a["ldx"], BYTES[a["dtype"]])
    holds("offsets", a["offsets"], a["groups"] + 1, 4)
    holds("source", a["source"], rows, 4)
    if a["Q"] is not None:
        result(a, ("Q", "S", "ldq", "lds"), rows, cols)
    if a["T"] is not None:
        result(a, ("T", "ST", "ldt", "ldst"), cols, X.mg_grouped_columns(rows, a["groups"]))


def grouped(a):
    rows, n, k = a["rows"], a["n"], a["k"]
    holds("offsets", a["offsets"], a["groups"] + 1, 4)
    holds("source", a["source"], rows, 4)
    result(a, ("A", "SA", "lda", "ldsa"), -(-rows // a["fan"]) if a["source"] is not None else rows, k)
    result(a, ("B", "SB", "ldb", "ldsb", "stride_b", "stride_sb"), n, k, True, a["groups"])
    matrix("C", a["C"], rows, n, a["ldc"], BYTES[a["c_type"]])


def grouped_sum(a):
    columns, m, n = X.mg_grouped_columns(a["rows"], a["groups"]), a["m"], a["n"]
    holds("offsets", a["offsets"], a["groups"] + 1, 4)
    result(a, ("A", "SA", "lda", "ldsa"), m, columns)
    result(a, ("B", "SB", "ldb", "ldsb"), n, columns)
    holds("C", a["C"], (a["groups"] - 1) * a["stride_c"] + (m - 1) * a["ldc"] + n, BYTES[a["c_type"]])


def sort(a):
    slots = a["tokens"] * a["fan"]
    for name, count in (("ids", slots), ("offsets", a["experts"] + 1), ("position", slots), ("source", slots)):
        holds(name, a[name], count, 4)
    assert a["ids"].dtype == torch.int32


def combine(a):
    z, slots, cols = BYTES[a["dtype"]], a["tokens"] * a["fan"], a["cols"]
    matrix("Y", a["Y"], slots, cols, a["ldy"], z)
    matrix("O", a["O"], a["tokens"], cols, a["ldo"], z)
    holds("position", a["position"], slots, 4)
    holds("weights", a["weights"], slots, 4)
    assert a["weights"] is None or a["weights"].dtype == torch.float32


def combine_grad(a):
    z, slots, cols = BYTES[a["dtype"]], a["tokens"] * a["fan"], a["cols"]
    matrix("dO", a["dO"], a["tokens"], cols, a["lddo"], z)
    matrix("Y", a["Y"], slots, cols, a["ldy"], z)
    matrix("dY", a["dY"], slots, cols, a["lddy"], z)
    for name in ("position", "weights", "dweights"):
        holds(name, a[name], slots, 4)
    assert a["weights"].dtype == torch.float32 and a["dweights"].dtype == torch.float32
    assert a["dO"].element_size() == a["Y"].element_size() == a["dY"].element_size() == z


CHECKS = {"mg_block_quantize": quantize, "mg_block_quantize_batched": quantize_batched, "mg_block_quantize_grouped": quantize_grouped, "mg_block_gemm_grouped": grouped,
          "mg_block_gemm_grouped_sum": grouped_sum, "mg_expert_sort": sort, "mg_expert_combine": combine, "mg_expert_combine_grad": combine_grad}


@pytest.fixture
def calls(monkeypatch):
    """the names of the calls so far; each has been looked over"""
    made = []

    def recorded(name, signature):
        def call(*args, **named):
            CHECKS[name](signature.bind(*args, **named).arguments)
            made.append(name)
            return 0
        return call
    for name in X._calls:
        signature = inspect.signature(getattr(X, name))
        monkeypatch.setattr(X, name, recorded(name, signature))
    with FakeTensorMode():
        yield made


def new(*shape, kind=torch.bfloat16, device="cuda"):
    return torch.empty(*shape, dtype=kind, device=device)


def layer(kind=torch.bfloat16):
    return L.ExpertLayer(new(EXPERTS, HIDDEN, WIDTH, kind=kind), new(EXPERTS, WIDTH, HIDDEN, kind=kind))


def given(kind=torch.bfloat16, gates=torch.float32, ids=torch.int64):
    return new(TOKENS, WIDTH, kind=kind), new(TOKENS, FAN, kind=ids), new(TOKENS, FAN, kind=gates)


@pytest.mark.parametrize("kind", (torch.float32, torch.float16, torch.bfloat16))
@pytest.mark.parametrize("gates", (torch.float32, torch.float16, torch.bfloat16))
@pytest.mark.parametrize("weights", (torch.float32, torch.bfloat16))
def test_types_that_are_taken(calls, kind, gates, weights):
    """the gates of a 16-bit softmax count as the FP32 numbers they are; their gradient is in FP32"""
    mine = layer(weights)
    y = mine.forward(*given(kind, gates))
    assert y.shape == (TOKENS, WIDTH) and y.dtype == kind
    dx, d_gates, dw1, dw2 = mine.backward(new(TOKENS, WIDTH, kind=kind))
    assert dx.shape == y.shape and dx.dtype == kind and d_gates.shape == (TOKENS, FAN) and d_gates.dtype == torch.float32
    assert dw1.shape == (EXPERTS, HIDDEN, WIDTH) and dw2.shape == (EXPERTS, WIDTH, HIDDEN) and dw1.dtype == dw2.dtype == torch.float32
    assert calls.count("mg_expert_combine_grad") == 1 and calls.count("mg_block_gemm_grouped_sum") == 2


@pytest.mark.parametrize("ids", (torch.uint8, torch.int16, torch.int32, torch.int64))
def test_whole_numbers_of_any_width(calls, ids):
    layer().forward(*given(ids=ids))
    assert "mg_expert_sort" in calls


@pytest.mark.parametrize("kind,dy", ((torch.bfloat16, torch.float32), (torch.float32, torch.bfloat16), (torch.float16, torch.bfloat16), (torch.bfloat16, torch.float64)))
def test_gradient_of_another_type_is_refused(calls, kind, dy):
    mine = layer()
    mine.forward(*given(kind))
    del calls[:]
    with pytest.raises(TypeError, match="dy"):
        mine.backward(new(TOKENS, WIDTH, kind=dy))
    assert not calls


@pytest.mark.parametrize("which,value", (
    ("x", (TOKENS, WIDTH - 1)), ("x", (TOKENS - 1, WIDTH)), ("x", (TOKENS + 1, WIDTH)), ("x", (TOKENS * WIDTH,)), ("x", (2, TOKENS // 2, WIDTH)),
    ("gates", (TOKENS, FAN - 1)), ("gates", (TOKENS - 1, FAN)), ("gates", (FAN, TOKENS)), ("gates", (TOKENS,)), ("ids", (TOKENS,)), ("ids", (TOKENS, FAN + 1))))
def test_shapes_that_do_not_fit_are_refused(calls, which, value):
    mine, args = layer(), dict(zip(("x", "ids", "gates"), given()))
    args[which] = new(*value, kind=args[which].dtype)
    del calls[:]
    with pytest.raises(ValueError, match="x|ids|gates"):
        mine.forward(**args)
    assert not calls


@pytest.mark.parametrize("which,kind", (("x", torch.float64), ("x", torch.int32), ("gates", torch.float64), ("gates", torch.int64), ("ids", torch.float32), ("ids", torch.bool)))
def test_types_that_are_refused(calls, which, kind):
    mine, args = layer(), dict(zip(("x", "ids", "gates"), given()))
    args[which] = new(*args[which].shape, kind=kind)
    del calls[:]
    with pytest.raises(TypeError, match=which):
        mine.forward(**args)
    assert not calls


@pytest.mark.parametrize("which", ("x", "ids", "gates", "dy"))
def test_host_memory_is_refused(calls, which):
    mine, args = layer(), dict(zip(("x", "ids", "gates"), given()))
    if which == "dy":
        mine.forward(**args)
        with pytest.raises(ValueError, match="dy"):
            mine.backward(new(TOKENS, WIDTH, device="cpu"))
        return
    args[which] = new(*args[which].shape, kind=args[which].dtype, device="cpu")
    with pytest.raises(ValueError, match=which):
        mine.forward(**args)


@pytest.mark.parametrize("shape", ((TOKENS, WIDTH + 1), (TOKENS - 1, WIDTH), (TOKENS * FAN, WIDTH), (TOKENS * WIDTH,)))
def test_gradient_of_another_shape_is_refused(calls, shape):
    mine = layer()
    mine.forward(*given())
    with pytest.raises(ValueError, match="dy"):
        mine.backward(new(*shape))


def test_weights_that_do_not_fit_are_refused(calls):
    w1, w2 = new(EXPERTS, HIDDEN, WIDTH), new(EXPERTS, WIDTH, HIDDEN)
    for a, b in ((w1, w1), (w1, w2[:-1]), (w1, w2[:, :-1]), (w1, w2[:, :, :-1]), (w1[0], w2[0])):
        with pytest.raises(ValueError):
            L.ExpertLayer(a, b)
    for a, b in ((w1.double(), w2.double()), (w1.int(), w2)):
        with pytest.raises(TypeError):
            L.ExpertLayer(a, b)
    with pytest.raises(ValueError):
        L.ExpertLayer(w1.cpu(), w2.cpu())


def test_products_by_themselves(calls):
    """Experts without the layer: rows of tokens or of routes, and the routes of as many experts"""
    part, routes = L.Experts(new(EXPERTS, HIDDEN, WIDTH)), L.Routes(new(TOKENS, FAN, kind=torch.int32), EXPERTS)
    x, rows, dy = new(TOKENS, WIDTH), new(TOKENS * FAN, WIDTH), new(TOKENS * FAN, HIDDEN)
    assert part.forward(routes, x, of_tokens=True).shape == (TOKENS * FAN, HIDDEN)
    assert part.forward(routes, new(WIDTH, TOKENS * FAN).t(), of_tokens=False).shape == (TOKENS * FAN, HIDDEN)
    for from_tokens, of_x in ((True, x), (False, rows)):
        dx, dw = part.backward(routes, of_x, from_tokens, dy)
        assert dx.shape == (TOKENS * FAN, WIDTH) and dw.shape == (EXPERTS, HIDDEN, WIDTH)
    del calls[:]
    for of_x, from_tokens in ((x, False), (rows, True), (x[:, :-1], True), (new(TOKENS, HIDDEN), True)):
        with pytest.raises(ValueError):
            part.forward(routes, of_x, from_tokens)
        with pytest.raises(ValueError):
            part.backward(routes, of_x, from_tokens, dy)
    for of_dy in (dy[:-1], dy[:, :-1], new(TOKENS, HIDDEN)):
        with pytest.raises(ValueError):
            part.backward(routes, x, True, of_dy)
    fewer = L.Routes(new(TOKENS, FAN, kind=torch.int32), EXPERTS - 1)
    with pytest.raises(ValueError):
        part.forward(fewer, x, True)
    part.weights = new(EXPERTS, HIDDEN, WIDTH - 1)
    with pytest.raises(ValueError):
        part.quantize()
    assert calls == ["mg_expert_sort"]


def test_no_tokens(calls):
    mine = layer()
    y = mine.forward(new(0, WIDTH), new(0, FAN, kind=torch.int64), new(0, FAN, kind=torch.float32))
    dx, d_gates, dw1, _ = mine.backward(y)
    assert y.shape == dx.shape == (0, WIDTH) and d_gates.shape == (0, FAN) and dw1.shape == (EXPERTS, HIDDEN, WIDTH)


@pytest.mark.parametrize("ids", INDEX_TYPES)
def test_ids_keep_their_meaning_in_32_bits(ids):
    """numbers that 32 bits cannot hold belong to no expert, as in 64 bits"""
    values = [0, 1, 4] + ([-1, -7] if ids != torch.uint8 else []) + ([5, 100] if ids.itemsize < 4 else [5, 1 << 20, (1 << 31) - 1])
    if ids == torch.int64:
        values += [1 << 31, 1 << 32, (1 << 32) + 1, -(1 << 32) + 2, (1 << 63) - 1, -(1 << 63)]
    given = torch.tensor(values, dtype=ids).view(-1, 1)
    got = L.dense_ids(given, EXPERTS)
    assert got.dtype == torch.int32 and got.shape == given.shape and got.is_contiguous()
    assert [v if 0 <= v < EXPERTS else None for v in got.view(-1).tolist()] == [v if 0 <= v < EXPERTS else None for v in values]


def test_memory_is_on_the_device_of_the_arguments(calls):
    """whatever that is called, and none of them mixed"""
    on = "cuda:1"
    mine = L.ExpertLayer(new(EXPERTS, HIDDEN, WIDTH, device=on), new(EXPERTS, WIDTH, HIDDEN, device=on))
    y = mine.forward(new(TOKENS, WIDTH, device=on), new(TOKENS, FAN, kind=torch.int64, device=on), new(TOKENS, FAN, device=on))
    parts = [y, *mine.backward(y), mine.up.w.q, mine.up.turned.s, mine.down.w.s]
    assert {str(t.device) for t in parts} == {on}
    with pytest.raises(ValueError, match="x"):
        mine.forward(new(TOKENS, WIDTH), new(TOKENS, FAN, kind=torch.int64, device=on), new(TOKENS, FAN, device=on))
    with pytest.raises(ValueError, match="x"):
        mine.up.forward(L.Routes(new(TOKENS, FAN, kind=torch.int32, device=on), EXPERTS), new(TOKENS, WIDTH), True)
    with pytest.raises(ValueError, match="weights"):
        mine.up.forward(L.Routes(new(TOKENS, FAN, kind=torch.int32), EXPERTS), new(TOKENS, WIDTH), True)


def test_a_served_call_keeps_nothing(calls):
    """neither its own activations nor an earlier call's, which would not belong to its answer"""
    mine = layer()
    mine.forward(*given())
    y = mine.forward(*given(), keep=False)
    assert mine.kept is None
    with pytest.raises(RuntimeError):
        mine.backward(y)
    mine.forward(*given())
    mine.backward(y)

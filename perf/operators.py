"""The 8-bit products and the routing of a mixture-of-experts layer: what programs ask of `paper_1705_05249_amd.experts`.

`listed()` names twelve calls, from the products of one token to a training step of the experts; `draw(rng)` gives more of the same ranges.
`prepare` makes what a program holds before the call, `run` is the call: with `own` through the library's entry points, otherwise the same
formulas in elementary torch operations, in FP32 with one rounding at the end.  `exact` computes the definitions once more in 64 bits.

Matrices are row-major.  An 8-bit matrix (e4m3: 4 bits of exponent, 3 of mantissa, largest value 448) has one FP32 scale for each block of 128
consecutive elements of a row, or for each block of 128 x 128; an element stands for its 8-bit value times its block's scale.  The scale that
quantising chooses is the smallest power of two (of 2^-126 at least; 1 for a block of zeros) with which the block's largest magnitude is at most 448.
"""
import math

import torch

own = False

BLOCK = 128
FP8 = torch.float8_e4m3fn
TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
SIZE = {"f32": 4, "f16": 2, "bf16": 2}
MOST_FLOPS = 6.0 * 16384 * 4096 * 2048      # of a drawn training step: the largest listed one
MOST_ELEMENTS = 8192 * 4096                 # of a drawn matrix that is quantised
MOST_ROUTED = 32768 * 4096                  # elements of the routed rows of a drawn call
MOST_WEIGHTS = 32 * 2048 * 4096             # elements of the weights of all experts of a drawn call


def listed():
    return [
        # a linear layer as it serves one token: the activations are quantised, the weights are a checkpoint's (any scales)
        dict(name="linear_1x4096x4096", routine="linear", m=1, n=4096, k=4096, dtype="bf16"),
        # the large square product of two 8-bit matrices with scales of any value
        dict(name="product_4096", routine="product", m=4096, n=4096, k=4096, scales="any", layout="row", b_block="square", odd_ld=False, dtype="bf16"),
        # sizes that are no multiple of any tile or block, rows that start at odd addresses
        dict(name="product_1000x1001x999", routine="product", m=1000, n=1001, k=999, scales="pow2", layout="col", b_block="row", odd_ld=True, dtype="f16"),
        # a training step of a linear layer: output, input's gradient, weights' gradient, with all quantising
        dict(name="linear_step_8192x4096x4096", routine="linear_step", m=8192, n=4096, k=4096, dtype="bf16"),
        # a few rows of activations: latency
        dict(name="quantize_64x1024", routine="quantize", rows=64, cols=1024, block="row", sides="plain", odd_ld=False, dtype="f16"),
        # activations of a batch for the forward product and, transposed, for the weights' gradient
        dict(name="quantize_8192x4096_both", routine="quantize", rows=8192, cols=4096, block="row", sides="both", odd_ld=False, dtype="bf16"),
        # eight tokens that are being generated, two experts each
        dict(name="sort_8x2_of_8", routine="sort", tokens=8, fan=2, experts=8, cols=4096, dtype="bf16"),
        # a long batch with many small experts; a capacity limit has dropped some tokens
        dict(name="sort_16384x8_of_64", routine="sort", tokens=16384, fan=8, experts=64, cols=2048, dtype="bf16"),
        # the experts' answers back to sixteen tokens
        dict(name="combine_16x2", routine="combine", tokens=16, fan=2, experts=8, cols=4096, dtype="f32"),
        # the same for a training batch, with the gradients of rows and weights
        dict(name="combine_step_8192x4", routine="combine_step", tokens=8192, fan=4, experts=32, cols=4096, dtype="bf16"),
        # experts that serve a few tokens each: their weights have to be read, little else
        dict(name="experts_24x4_of_32", routine="experts", tokens=24, fan=4, experts=32, n=2048, k=4096, dtype="bf16"),
        # a training step of the experts' products, with all quantising
        dict(name="experts_step_8192x2_of_16", routine="experts_step", tokens=8192, fan=2, experts=16, n=4096, k=2048, dtype="bf16"),
    ]


# ------------------------------------------------------------------------------------------------ drawn cases

def _size(rng, lo, hi, unit=64):
    """spread over the logarithm of lo .. hi; half are multiples of `unit`"""
    v = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    if v >= unit and rng.random() < 0.5:
        v = v // unit * unit
    return max(lo, min(hi, v))


def draw(rng):
    routine = rng.choice(("linear", "product", "product", "linear_step", "quantize", "sort", "combine", "combine_step", "experts", "experts_step"))
    dtype = rng.choice(("bf16", "bf16", "f16", "f32"))
    while True:
        case = _drawn(rng, routine, dtype)
        if case is not None:
            return case


def _drawn(rng, routine, dtype):
    if routine == "linear":
        return dict(routine=routine, m=_size(rng, 1, 64, 8), n=_size(rng, 256, 8192), k=_size(rng, 256, 8192), dtype=dtype)
    if routine == "product":
        m, n, k = (_size(rng, 16, 8192) for _ in range(3))
        case = dict(routine=routine, m=m, n=n, k=k, scales=rng.choice(("any", "pow2")), layout=rng.choice(("row", "col")),
                    b_block=rng.choice(("row", "square")), odd_ld=rng.random() < 0.3, dtype=dtype)
        return case if 2.0 * m * n * k <= MOST_FLOPS / 3 else None
    if routine == "linear_step":
        m, n, k = _size(rng, 32, 16384), _size(rng, 128, 8192), _size(rng, 128, 8192)
        return dict(routine=routine, m=m, n=n, k=k, dtype=dtype) if 6.0 * m * n * k <= MOST_FLOPS and max(m * n, m * k, n * k) <= MOST_ELEMENTS else None
    if routine == "quantize":
        rows, cols = _size(rng, 1, 32768), _size(rng, 64, 16384)
        case = dict(routine=routine, rows=rows, cols=cols, block=rng.choice(("row", "square")), sides=rng.choice(("plain", "turned", "both")),
                    odd_ld=rng.random() < 0.3, dtype=dtype)
        return case if rows * cols <= MOST_ELEMENTS else None
    experts = _size(rng, 2, 256, 8)
    fan = rng.randint(1, min(8, experts))
    if routine in ("sort", "combine", "combine_step"):
        tokens, cols = _size(rng, 1, 32768), _size(rng, 64, 8192)
        return dict(routine=routine, tokens=tokens, fan=fan, experts=experts, cols=cols, dtype=dtype) if tokens * fan * cols <= MOST_ROUTED else None
    n, k = _size(rng, 128, 4096), _size(rng, 128, 4096)
    tokens = _size(rng, 1, 256) if routine == "experts" else _size(rng, 64, 8192)
    if experts * n * k > MOST_WEIGHTS or 6.0 * tokens * fan * n * k > MOST_FLOPS:
        return None
    return dict(routine=routine, tokens=tokens, fan=fan, experts=experts, n=n, k=k, dtype=dtype)


# ------------------------------------------------------------------------------------------------ sizes

def _blocks(size):
    return -(-size // BLOCK)


def _ld(size, odd, piece=16):
    """a row's length in memory: whole 16-byte pieces, or a part of a larger matrix that starts anywhere"""
    return size + 7 - size % 2 if odd else -(-size // piece) * piece


def _columns(rows, groups):
    """columns of a turned 8-bit matrix of `rows` routed rows: each expert's start on a block of their own"""
    return _blocks(rows) * BLOCK + groups * BLOCK


# ------------------------------------------------------------------------------------------------ quantising, plainly

def _largest(x, block):
    """largest magnitude of each block of x (rows x cols): rows x blocks, or blocks x blocks"""
    rows, cols = x.shape
    tall = BLOCK if block == "square" else 1
    full = torch.nn.functional.pad(x.abs(), (0, -cols % BLOCK, 0, -rows % tall))
    return full.view(-1, tall, full.shape[1] // BLOCK, BLOCK).amax((1, 3))


def _spread(scales, rows, cols, block):
    """the scale of every element"""
    if block == "square":
        scales = scales.repeat_interleave(BLOCK, 0)[:rows]
    return scales.repeat_interleave(BLOCK, 1)[:, :cols]


def _quantize(x, block):
    """(8-bit matrix, scales) of x (rows x cols), in FP32"""
    x = x.float()
    largest = _largest(x, block)
    part, power = torch.frexp(largest)                          # largest = part * 2^power, 1/2 <= part < 1; 448 = 7/8 * 2^9
    power = torch.where(part > 0.875, power - 8, power - 9).clamp(min=-126)
    scales = torch.where(largest > 0, torch.ldexp(torch.ones_like(largest), power), torch.ones_like(largest))
    return (x / _spread(scales, *x.shape, block)).to(FP8), scales


def _values(q, scales, block):
    """what an 8-bit matrix stands for, in FP32"""
    return q.float() * _spread(scales, *q.shape, block)


def _rounded(x, block):
    q, scales = _quantize(x, block)
    return _values(q, scales, block)


# ------------------------------------------------------------------------------------------------ inputs

class _Draw:
    """activations and gradients with a few large channels, weights of variance 1 / k, the answers of a router"""

    def __init__(self, seed):
        self.gen = torch.Generator(device="cuda").manual_seed(seed)

    def normal(self, *shape, sigma=1.0):
        return torch.empty(shape, device="cuda").normal_(0.0, sigma, generator=self.gen)

    def activations(self, rows, cols, dtype, sigma=1.0):
        channels = torch.exp(self.normal(cols, sigma=0.8))
        return (self.normal(rows, cols, sigma=sigma) * channels).to(TYPES[dtype])

    def weights(self, *shape, dtype):
        return self.normal(*shape, sigma=shape[-1] ** -0.5).to(TYPES[dtype])

    def routes(self, tokens, fan, experts, dropped=0.0):
        """experts of every token (int32, -1: dropped) and the weights of their answers; some experts are asked far more often than others"""
        scores = self.normal(tokens, experts) + self.normal(experts)
        best, ids = torch.topk(scores, fan, dim=1)
        ids = ids.int()
        if dropped:
            ids[torch.rand((tokens, fan), device="cuda", generator=self.gen) < dropped] = -1
        return ids, torch.softmax(best, 1)

    def stored(self, x, ld):
        """x (rows x cols) in memory with rows `ld` elements apart"""
        held = torch.zeros((x.shape[0], ld), dtype=x.dtype, device="cuda")
        held[:, :x.shape[1]] = x
        return held


def _order(ids, experts):
    """(offsets, position, source) of routes: slots sorted by expert, in their own order within one; dropped ones last"""
    key = ids.reshape(-1).long()
    key = torch.where((key >= 0) & (key < experts), key, experts)
    source = torch.sort(key, stable=True)[1]
    position = torch.empty_like(source)
    position[source] = torch.arange(source.numel(), device="cuda")
    ends = (key[:, None] == torch.arange(experts, device="cuda")).sum(0).cumsum(0)
    offsets = torch.cat((torch.zeros_like(ends[:1]), ends))
    kept = torch.arange(source.numel(), device="cuda") < offsets[-1]
    position = torch.where(key < experts, position, -1)
    return offsets.int(), position.int(), torch.where(kept, source, -1).int()


def prepare(case, seed):
    s = dict(case)
    d, routine, dtype = _Draw(seed), case["routine"], case["dtype"]
    new = lambda *shape, kind=None: torch.empty(shape, dtype=kind or TYPES[dtype], device="cuda")  # noqa: E731
    byte = torch.uint8
    if routine in ("linear", "linear_step"):
        m, n, k = case["m"], case["n"], case["k"]
        s["x"] = d.activations(m, k, dtype)
        w = d.weights(n, k, dtype=dtype)
        if routine == "linear":
            # a checkpoint: scales of any value
            scales = _largest(w.float(), "square") / 448.0
            q = (w.float() / _spread(scales, n, k, "square")).to(FP8)
            s["w"], s["sw"], s["y"] = d.stored(q.view(byte), _ld(k, False)).view(FP8), scales, new(m, n)
        else:
            s["w"], s["dy"] = w, d.activations(m, n, dtype, sigma=1e-3)
            s["y"], s["dx"], s["dw"] = new(m, n), new(m, k), new(n, k, kind=torch.float32)
            s["wq"], s["wt"] = new(n, _ld(k, False), kind=byte), new(k, _ld(n, False), kind=byte)
            s["sw"], s["st"] = new(_blocks(n), _blocks(k), kind=torch.float32), new(_blocks(k), _blocks(n), kind=torch.float32)
            s["xt"], s["sxt"] = new(k, _ld(m, False), kind=byte), new(k, _blocks(m), kind=torch.float32)
            s["dq"], s["sd"] = new(m, _ld(n, False), kind=byte), new(m, _blocks(n), kind=torch.float32)
            s["dt"], s["sdt"] = new(n, _ld(m, False), kind=byte), new(n, _blocks(m), kind=torch.float32)
        s["xq"], s["sx"] = new(m, _ld(k, False), kind=byte), new(m, _blocks(k), kind=torch.float32)
    elif routine == "product":
        m, n, k = case["m"], case["n"], case["k"]
        lead = _ld(k, case["odd_ld"])
        for name, rows, block in (("a", m, "row"), ("b", n, case["b_block"])):
            q, scales = _quantize(d.activations(rows, k, "f32"), block)
            if case["scales"] == "any":
                scales = scales * torch.empty_like(scales).uniform_(0.5, 1.5, generator=d.gen)
            s[name], s["s" + name] = d.stored(q.view(byte), lead).view(FP8), scales
        s["c"] = new(m, n) if case["layout"] == "row" else new(n, m)
    elif routine == "quantize":
        rows, cols = case["rows"], case["cols"]
        s["x"] = d.stored(d.activations(rows, cols, dtype), _ld(cols, case["odd_ld"], 8))
        tall, wide = (_blocks(rows), _blocks(cols)) if case["block"] == "square" else (rows, cols)
        s["q"] = new(rows, _ld(cols, case["odd_ld"]), kind=byte) if case["sides"] != "turned" else None
        s["s"] = new(tall, _blocks(cols), kind=torch.float32) if case["sides"] != "turned" else None
        s["t"] = new(cols, _ld(rows, case["odd_ld"]), kind=byte) if case["sides"] != "plain" else None
        s["st"] = new(wide, _blocks(rows), kind=torch.float32) if case["sides"] != "plain" else None
    else:
        tokens, fan, experts = case["tokens"], case["fan"], case["experts"]
        rows = tokens * fan
        training = routine in ("sort", "combine", "combine_step")
        ids, s["gates"] = d.routes(tokens, fan, experts, dropped=0.02 if training and tokens >= 256 else 0.0)
        if routine == "sort":
            s["ids"], s["x"] = ids, d.activations(tokens, case["cols"], dtype)
            s["offsets"], s["position"], s["source"] = (new(c, kind=torch.int32) for c in (experts + 1, rows, rows))
            s["out"] = new(rows, case["cols"])
        else:
            s["offsets"], s["position"], s["source"] = _order(ids, experts)
        if routine in ("combine", "combine_step"):
            s["y"], s["out"] = d.activations(rows, case["cols"], dtype), new(tokens, case["cols"])
            if routine == "combine_step":
                s["dout"] = d.activations(tokens, case["cols"], dtype, sigma=1e-3)
                s["dy"], s["dgates"] = torch.zeros_like(s["y"]), new(tokens, fan, kind=torch.float32)
        elif routine in ("experts", "experts_step"):
            n, k = case["n"], case["k"]
            s["x"] = d.activations(tokens, k, dtype)
            w = d.weights(experts, n, k, dtype=dtype)
            s["xq"], s["sx"] = new(tokens, _ld(k, False), kind=byte), new(tokens, _blocks(k), kind=torch.float32)
            s["y"] = new(rows, n)
            s["wq"], s["sw"] = new(experts, n, _ld(k, False), kind=byte), new(experts, _blocks(n), _blocks(k), kind=torch.float32)
            if routine == "experts":
                # quantised once, when the weights were loaded
                for e in range(experts):
                    q, s["sw"][e] = _quantize(w[e], "square")
                    s["wq"][e, :, :k] = q.view(byte)
            else:
                columns = _columns(rows, experts)
                s["w"], s["dy"] = w, d.activations(rows, n, dtype, sigma=1e-3)
                s["dx"], s["dw"] = new(rows, k), new(experts, n, k, kind=torch.float32)
                s["wt"], s["st"] = new(experts, k, _ld(n, False), kind=byte), new(experts, _blocks(k), _blocks(n), kind=torch.float32)
                s["xt"], s["sxt"] = new(k, columns, kind=byte), new(k, columns // BLOCK, kind=torch.float32)
                s["dq"], s["sd"] = new(rows, _ld(n, False), kind=byte), new(rows, _blocks(n), kind=torch.float32)
                s["dt"], s["sdt"] = new(n, columns, kind=byte), new(n, columns // BLOCK, kind=torch.float32)
    _workspaces(s)
    return s


def _workspaces(s):
    """what the library asks a program to keep for a call, as bytes of scratch memory"""
    s["ws"] = None
    try:
        from paper_1705_05249_amd import experts as X
    except ImportError:                      # the plain forms need none
        return
    routine = s["routine"]
    if routine == "sort":
        count = X.mg_expert_sort_workspace_bytes(s["tokens"], s["fan"], s["experts"])
    elif routine in ("linear", "product"):
        count = X.mg_block_gemm_workspace_bytes(s["m"], s["n"], s["k"])
    elif routine == "linear_step":
        m, n, k = s["m"], s["n"], s["k"]
        count = max(X.mg_block_gemm_workspace_bytes(*size) for size in ((m, n, k), (m, k, n), (n, k, m)))
    elif routine in ("experts", "experts_step"):
        experts, rows, n, k = s["experts"], s["tokens"] * s["fan"], s["n"], s["k"]
        count = X.mg_block_gemm_grouped_workspace_bytes(experts, rows, n, k)
        if routine == "experts_step":
            count = max(count, X.mg_block_gemm_grouped_workspace_bytes(experts, rows, k, n), X.mg_block_gemm_grouped_sum_workspace_bytes(experts, rows, n, k))
    else:
        return
    s["ws"] = torch.empty(count, dtype=torch.uint8, device="cuda") if count else None


# ------------------------------------------------------------------------------------------------ the calls

def run(s):
    return (_OWN if own else _PLAIN)[s["routine"]](s)


def _codes(s):
    from paper_1705_05249_amd import experts as X
    return X, {"f32": X.MG_F32, "f16": X.MG_F16, "bf16": X.MG_BF16}[s["dtype"]]


def _own_linear(s):
    X, code = _codes(s)
    m, n, k = s["m"], s["n"], s["k"]
    lead, blocks = s["xq"].stride(0), s["sx"].stride(0)
    X.mg_block_quantize(code, X.MG_BLOCK_ROW, m, k, s["x"], k, s["xq"], lead, s["sx"], blocks, None, 0, None, 0)
    X.mg_block_gemm(X.MG_ROW_MAJOR, m, n, k, 1.0, X.MG_SCALES_ANY, X.MG_BLOCK_ROW, s["xq"], lead, s["sx"], blocks,
                    X.MG_BLOCK_SQUARE, s["w"], s["w"].stride(0), s["sw"], s["sw"].stride(0), 0.0, code, s["y"], n, s["ws"])
    return s["y"]


def _own_product(s):
    X, code = _codes(s)
    m, n, k, row = s["m"], s["n"], s["k"], s["layout"] == "row"
    X.mg_block_gemm(X.MG_ROW_MAJOR if row else X.MG_COL_MAJOR, m, n, k, 1.0, X.MG_SCALES_ANY if s["scales"] == "any" else X.MG_SCALES_POW2,
                    X.MG_BLOCK_ROW, s["a"], s["a"].stride(0), s["sa"], s["sa"].stride(0),
                    X.MG_BLOCK_ROW if s["b_block"] == "row" else X.MG_BLOCK_SQUARE, s["b"], s["b"].stride(0), s["sb"], s["sb"].stride(0),
                    0.0, code, s["c"], s["c"].stride(0), s["ws"])
    return s["c"]


def _own_linear_step(s):
    X, code = _codes(s)
    m, n, k = s["m"], s["n"], s["k"]
    at = lambda name, scales: (s[name], s[name].stride(0), s[scales], s[scales].stride(0))  # noqa: E731
    ROW, SQUARE, P = X.MG_BLOCK_ROW, X.MG_BLOCK_SQUARE, X.MG_SCALES_POW2
    X.mg_block_quantize(code, ROW, m, k, s["x"], k, *at("xq", "sx"), *at("xt", "sxt"))
    X.mg_block_quantize(code, SQUARE, n, k, s["w"], k, *at("wq", "sw"), *at("wt", "st"))
    X.mg_block_quantize(code, ROW, m, n, s["dy"], n, *at("dq", "sd"), *at("dt", "sdt"))
    X.mg_block_gemm(X.MG_ROW_MAJOR, m, n, k, 1.0, P, ROW, *at("xq", "sx"), SQUARE, *at("wq", "sw"), 0.0, code, s["y"], n, s["ws"])
    X.mg_block_gemm(X.MG_ROW_MAJOR, m, k, n, 1.0, P, ROW, *at("dq", "sd"), SQUARE, *at("wt", "st"), 0.0, code, s["dx"], k, s["ws"])
    X.mg_block_gemm(X.MG_ROW_MAJOR, n, k, m, 1.0, P, ROW, *at("dt", "sdt"), ROW, *at("xt", "sxt"), 0.0, X.MG_F32, s["dw"], k, s["ws"])
    return s["y"], s["dx"], s["dw"]


def _own_quantize(s):
    X, code = _codes(s)
    rows, cols = s["rows"], s["cols"]
    at = lambda name, scales: (None, 0, None, 0) if s[name] is None else (s[name], s[name].stride(0), s[scales], s[scales].stride(0))  # noqa: E731
    X.mg_block_quantize(code, X.MG_BLOCK_ROW if s["block"] == "row" else X.MG_BLOCK_SQUARE, rows, cols, s["x"], s["x"].stride(0), *at("q", "s"), *at("t", "st"))
    return [None if s[name] is None else s[name].view(FP8)[:, :width] for name, width in (("q", cols), ("t", rows))] + [s["s"], s["st"]]


def _own_sort(s):
    X, code = _codes(s)
    tokens, fan, cols = s["tokens"], s["fan"], s["cols"]
    X.mg_expert_sort(tokens, fan, s["experts"], s["ids"], s["offsets"], s["position"], s["source"], s["ws"])
    X.mg_expert_gather(code, tokens, fan, cols, s["x"], cols, s["source"], None, s["out"], cols)
    return s["offsets"], s["position"], s["source"], s["out"]


def _own_combine(s):
    X, code = _codes(s)
    X.mg_expert_combine(code, s["tokens"], s["fan"], s["cols"], s["y"], s["cols"], s["position"], s["gates"], s["out"], s["cols"])
    return s["out"]


def _own_combine_step(s):
    X, code = _codes(s)
    cols = s["cols"]
    _own_combine(s)
    X.mg_expert_combine_grad(code, s["tokens"], s["fan"], cols, s["dout"], cols, s["y"], cols, s["position"], s["gates"], s["dy"], cols, s["dgates"])
    return s["out"], s["dy"], s["dgates"]


def _own_experts(s):
    X, code = _codes(s)
    tokens, fan, experts, n, k = s["tokens"], s["fan"], s["experts"], s["n"], s["k"]
    lead, blocks, lead_w = s["xq"].stride(0), s["sx"].stride(0), s["wq"].stride(1)
    X.mg_block_quantize(code, X.MG_BLOCK_ROW, tokens, k, s["x"], k, s["xq"], lead, s["sx"], blocks, None, 0, None, 0)
    X.mg_block_gemm_grouped(experts, s["offsets"], tokens * fan, n, k, 1.0, X.MG_SCALES_POW2, s["xq"], lead, s["sx"], blocks, s["source"], fan,
                            X.MG_BLOCK_SQUARE, s["wq"], lead_w, s["wq"].stride(0), s["sw"], s["sw"].stride(1), s["sw"].stride(0), 0.0, code, s["y"], n, s["ws"])
    return s["y"]


def _own_experts_step(s):
    X, code = _codes(s)
    tokens, fan, experts, n, k = s["tokens"], s["fan"], s["experts"], s["n"], s["k"]
    rows, offsets = tokens * fan, s["offsets"]
    at = lambda name, scales: (s[name], s[name].stride(0), s[scales], s[scales].stride(0))  # noqa: E731
    each = lambda name, scales: (s[name], s[name].stride(1), s[name].stride(0), s[scales], s[scales].stride(1), s[scales].stride(0))  # noqa: E731
    ROW, SQUARE, P, none = X.MG_BLOCK_ROW, X.MG_BLOCK_SQUARE, X.MG_SCALES_POW2, (None, 0, None, 0)
    X.mg_block_quantize_batched(code, SQUARE, experts, n, k, s["w"], k, n * k, *each("wq", "sw"), *each("wt", "st"))
    X.mg_block_quantize(code, ROW, tokens, k, s["x"], k, *at("xq", "sx"), *none)
    X.mg_block_quantize_grouped(code, experts, offsets, rows, k, s["x"], k, s["source"], fan, *none, *at("xt", "sxt"))
    X.mg_block_quantize_grouped(code, experts, offsets, rows, n, s["dy"], n, None, 1, *at("dq", "sd"), *at("dt", "sdt"))
    X.mg_block_gemm_grouped(experts, offsets, rows, n, k, 1.0, P, *at("xq", "sx"), s["source"], fan, SQUARE, *each("wq", "sw"), 0.0, code, s["y"], n,
                            s["ws"])
    X.mg_block_gemm_grouped(experts, offsets, rows, k, n, 1.0, P, *at("dq", "sd"), None, 1, SQUARE, *each("wt", "st"), 0.0, code, s["dx"], k, s["ws"])
    X.mg_block_gemm_grouped_sum(experts, offsets, rows, n, k, 1.0, P, *at("dt", "sdt"), *at("xt", "sxt"), 0.0, X.MG_F32, s["dw"], k, n * k, s["ws"])
    return s["y"], s["dx"], s["dw"]


_OWN = {"linear": _own_linear, "product": _own_product, "linear_step": _own_linear_step, "quantize": _own_quantize, "sort": _own_sort,
        "combine": _own_combine, "combine_step": _own_combine_step, "experts": _own_experts, "experts_step": _own_experts_step}


# ------------------------------------------------------------------------------------------------ the same, plainly

def _plain_linear(s):
    return (_rounded(s["x"], "row") @ _values(s["w"][:, :s["k"]], s["sw"], "square").T).to(TYPES[s["dtype"]])


def _plain_product(s):
    k = s["k"]
    a, b = _values(s["a"][:, :k], s["sa"], "row"), _values(s["b"][:, :k], s["sb"], s["b_block"])
    return (a @ b.T if s["layout"] == "row" else b @ a.T).to(TYPES[s["dtype"]])


def _plain_linear_step(s):
    kind = TYPES[s["dtype"]]
    w, x, dy = _rounded(s["w"], "square"), s["x"], s["dy"]
    y = (_rounded(x, "row") @ w.T).to(kind)
    dx = (_rounded(dy, "row") @ w).to(kind)
    return y, dx, _rounded(dy.T, "row") @ _rounded(x.T, "row").T


def _plain_quantize(s):
    x = s["x"][:, :s["cols"]]
    q, scales = _quantize(x, s["block"]) if s["q"] is not None else (None, None)
    t, turned = _quantize(x.T, s["block"]) if s["t"] is not None else (None, None)
    return [q, t, scales, turned]


def _plain_sort(s):
    offsets, position, source = _order(s["ids"], s["experts"])
    rows = s["x"][(source // s["fan"]).clamp(min=0)]
    return offsets, position, source, torch.where(source[:, None] >= 0, rows, 0)


def _answers(s):
    """the experts' answers in the order of the tokens, tokens x fan x cols in FP32; zeros for dropped ones"""
    at = s["position"].view(s["tokens"], s["fan"])
    return torch.where(at[:, :, None] >= 0, s["y"][at.clamp(min=0)].float(), 0.0)


def _plain_combine(s):
    return (_answers(s) * s["gates"][:, :, None]).sum(1).to(TYPES[s["dtype"]])


def _plain_combine_step(s):
    answers, dout, at = _answers(s), s["dout"].float(), s["position"]
    out = (answers * s["gates"][:, :, None]).sum(1).to(TYPES[s["dtype"]])
    rows = (s["gates"][:, :, None] * dout[:, None, :]).to(TYPES[s["dtype"]]).view(-1, s["cols"])
    dy = torch.zeros_like(torch.cat((s["y"], s["y"][:1])))      # (the last row: where the dropped ones go)
    dy[torch.where(at >= 0, at, at.numel())] = rows
    return out, dy[:-1], (answers * dout[:, None, :]).sum(2)


def _by_expert(s, rows, weights):
    """rows of each expert times its weights (experts x k x n); one product for each expert, their sizes as they are"""
    counts = (s["offsets"][1:] - s["offsets"][:-1]).tolist()
    return torch.cat([part @ w for part, w in zip(rows.split(counts), weights)])


def _rounded_weights(w):
    experts, n, k = w.shape
    if n % BLOCK == 0:
        return _rounded(w.reshape(-1, k), "square").view(experts, n, k)
    padded = torch.nn.functional.pad(w.float(), (0, 0, 0, -n % BLOCK))
    return _rounded(padded.view(-1, k), "square").view(experts, -1, k)[:, :n]


def _plain_experts(s):
    experts, n, k = s["experts"], s["n"], s["k"]
    spread = s["sw"].repeat_interleave(BLOCK, 1)[:, :n].repeat_interleave(BLOCK, 2)[:, :, :k]
    w = s["wq"].view(FP8)[:, :, :k].float() * spread
    x = _rounded(s["x"], "row")[s["source"] // s["fan"]]
    return _by_expert(s, x, w.transpose(1, 2)).to(TYPES[s["dtype"]])


def _plain_experts_step(s):
    kind, counts = TYPES[s["dtype"]], (s["offsets"][1:] - s["offsets"][:-1]).tolist()
    w = _rounded_weights(s["w"])
    rows = s["x"][s["source"] // s["fan"]]
    y = _by_expert(s, _rounded(s["x"], "row")[s["source"] // s["fan"]], w.transpose(1, 2)).to(kind)
    dx = _by_expert(s, _rounded(s["dy"], "row"), w).to(kind)
    dw = torch.stack([_turned(d) @ _turned(x).T for d, x in zip(s["dy"].split(counts), rows.split(counts))])
    return y, dx, dw


def _turned(x):
    """x^T, quantised in blocks of 128 rows of x (an expert without rows has none)"""
    return _rounded(x.T, "row") if x.shape[0] else x.T.float()


_PLAIN = {"linear": _plain_linear, "product": _plain_product, "linear_step": _plain_linear_step, "quantize": _plain_quantize, "sort": _plain_sort,
          "combine": _plain_combine, "combine_step": _plain_combine_step, "experts": _plain_experts, "experts_step": _plain_experts_step}


# ------------------------------------------------------------------------------------------------ 64 bits

def _exact_quantize(x, block):
    """(values of the 8-bit numbers, scales) by the definition: round to a multiple of the step of the number's binade, ties to even"""
    x = x.double()
    rows, cols = x.shape
    tall = BLOCK if block == "square" else 1
    r, c = torch.arange(rows, device=x.device) // tall, torch.arange(cols, device=x.device) // BLOCK
    wide = torch.zeros(rows, _blocks(cols), dtype=torch.float64, device=x.device).index_reduce_(1, c, x.abs(), "amax")
    largest = torch.zeros(-(-rows // tall), _blocks(cols), dtype=torch.float64, device=x.device).index_reduce_(0, r, wide, "amax")
    scales = torch.exp2(torch.ceil(torch.log2(torch.where(largest > 0, largest / 448, 1.0))).clamp(min=-126))
    v = x / scales[r][:, c]
    step = torch.exp2(torch.floor(torch.log2(v.abs().clamp(min=2.0 ** -6))) - 3)
    return torch.round(v / step) * step, scales


def _exact_rounded(x, block):
    v, scales = _exact_quantize(x, block)
    tall = BLOCK if block == "square" else 1
    r, c = torch.arange(x.shape[0], device=x.device) // tall, torch.arange(x.shape[1], device=x.device) // BLOCK
    return v * scales[r][:, c]


def _exact_values(q, scales, block):
    tall = BLOCK if block == "square" else 1
    r, c = torch.arange(q.shape[0], device=q.device) // tall, torch.arange(q.shape[1], device=q.device) // BLOCK
    return q.double() * scales.double()[r][:, c]


def exact(case, seed):
    s = prepare(case, seed)
    routine = case["routine"]
    if routine == "linear":
        return _exact_rounded(s["x"], "row") @ _exact_values(s["w"][:, :s["k"]], s["sw"], "square").T
    if routine == "product":
        a, b = (_exact_values(s[name][:, :s["k"]], s["s" + name], block) for name, block in (("a", "row"), ("b", s["b_block"])))
        return a @ b.T if s["layout"] == "row" else b @ a.T
    if routine == "linear_step":
        x, w, dy = s["x"], _exact_rounded(s["w"], "square"), s["dy"]
        return (_exact_rounded(x, "row") @ w.T, _exact_rounded(dy, "row") @ w,
                _exact_rounded(dy.T, "row") @ _exact_rounded(x.T, "row").T)
    if routine == "quantize":
        x = s["x"][:, :s["cols"]]
        q, scales = _exact_quantize(x, s["block"]) if s["q"] is not None else (None, None)
        t, turned = _exact_quantize(x.T, s["block"]) if s["t"] is not None else (None, None)
        return [q, t, scales, turned]
    if routine == "sort":
        ids = s["ids"].reshape(-1).tolist()
        kept = sorted((e, i) for i, e in enumerate(ids) if 0 <= e < s["experts"])
        out = torch.zeros(len(ids), s["cols"], dtype=torch.float64, device="cuda")
        if kept:
            out[:len(kept)] = s["x"].double()[torch.tensor([i // s["fan"] for _, i in kept], device="cuda")]
        return None, None, None, out
    if routine in ("combine", "combine_step"):
        out = torch.zeros(s["tokens"], s["cols"], dtype=torch.float64, device="cuda")
        dy, dgates = torch.zeros(s["y"].shape, dtype=torch.float64, device="cuda"), torch.zeros(s["gates"].shape, dtype=torch.float64, device="cuda")
        for j in range(s["fan"]):
            at = s["position"].view(-1, s["fan"])[:, j].long()
            here = (at >= 0).nonzero()[:, 0]
            rows, gate = s["y"].double()[at[here]], s["gates"].double()[here, j]
            out[here] += gate[:, None] * rows
            if routine == "combine_step":
                dout = s["dout"].double()[here]
                dy[at[here]] = gate[:, None] * dout
                dgates[here, j] = (rows * dout).sum(1)
        return out if routine == "combine" else (out, dy, dgates)
    offsets, token = s["offsets"].tolist(), s["source"].long() // s["fan"]
    y = torch.zeros(s["y"].shape, dtype=torch.float64, device="cuda")
    x = _exact_rounded(s["x"], "row")[token]
    training = routine == "experts_step"
    if training:
        dx, dw = torch.zeros(s["dx"].shape, dtype=torch.float64, device="cuda"), torch.zeros(s["dw"].shape, dtype=torch.float64, device="cuda")
        given = s["x"][token]
    for e in range(s["experts"]):
        lo, hi = offsets[e], offsets[e + 1]
        if lo == hi:
            continue
        w = _exact_rounded(s["w"][e], "square") if training else _exact_values(s["wq"][e].view(FP8)[:, :s["k"]], s["sw"][e], "square")
        y[lo:hi] = x[lo:hi] @ w.T
        if training:
            d = s["dy"][lo:hi]
            dx[lo:hi] = _exact_rounded(d, "row") @ w
            dw[e] = _exact_rounded(d.T, "row") @ _exact_rounded(given[lo:hi].T, "row").T
    return (y, dx, dw) if training else y


# ------------------------------------------------------------------------------------------------ what a call cannot do without

def work(case):
    """each input read once, each output written once; an 8-bit matrix that the call itself makes and reads is written once and read once"""
    routine, z = case["routine"], SIZE[case["dtype"]]
    if routine in ("linear", "product", "linear_step"):
        m, n, k = case["m"], case["n"], case["k"]
        if routine == "linear":
            return {"bytes": m * k * z + 2 * m * k + n * k + m * n * z, "flops": 2.0 * m * n * k}
        if routine == "product":
            return {"bytes": m * k + n * k + m * n * z, "flops": 2.0 * m * n * k}
        return {"bytes": (m * k + n * k + m * n) * (z + 4) + (m * n + m * k) * z + 4 * n * k, "flops": 6.0 * m * n * k}
    if routine == "quantize":
        return {"bytes": case["rows"] * case["cols"] * (z + (2 if case["sides"] == "both" else 1)), "flops": 0}
    tokens, rows = case["tokens"], case["tokens"] * case["fan"]
    if routine == "sort":
        return {"bytes": 12 * rows + (tokens + rows) * case["cols"] * z, "flops": 0}
    if routine == "combine":
        return {"bytes": 8 * rows + (tokens + rows) * case["cols"] * z, "flops": 2.0 * rows * case["cols"]}
    if routine == "combine_step":
        return {"bytes": 20 * rows + (2 * tokens + 2 * rows) * case["cols"] * z, "flops": 5.0 * rows * case["cols"]}
    experts, n, k = case["experts"], case["n"], case["k"]
    if routine == "experts":                     # the weights of experts that nobody asked are not read
        return {"bytes": tokens * k * (z + 2) + min(experts, rows) * n * k + rows * n * z, "flops": 2.0 * rows * n * k}
    weights = experts * n * k
    return {"bytes": weights * (z + 4 + 4) + tokens * k * (z + 2) + 2 * rows * k + rows * n * (z + 4) + rows * (n + k) * z, "flops": 6.0 * rows * n * k}

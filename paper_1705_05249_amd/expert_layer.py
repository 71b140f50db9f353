"""A mixture-of-experts layer on the entry points of experts.py: forward and backward pass with 8-bit products, and one token as it is served.

    y[t] = sum over j of gates[t, j] * W2[e] act(W1[e] x[t]),  e = ids[t, j],  act(h) = max(h, 0)^2

    python -m paper_1705_05249_amd.expert_layer [tokens] [width] [hidden] [experts] [fan]

trains a layer to answer as another one does and prints the loss and the time of a step.  PyTorch holds the memory, computes the elementwise
activation and makes the update; everything else runs in the library's kernels.  All buffers are allocated by the layer, on
its weights' device, none by the library; the calls go to torch's current stream, so that device has to be the current one.
Rows of 16 bits are products on the FP8 matrix pipes, whose sums have fewer bits than FP32 (MG_SUMS_FP32 in include/mg_experts.h says how many);
rows in FP32 and the weights' gradients are summed in FP32.
"""
import sys

import torch

from . import experts as X

TYPES = {torch.float32: X.MG_F32, torch.float16: X.MG_F16, torch.bfloat16: X.MG_BF16}
INDEX_TYPES = (torch.uint8, torch.int8, torch.int16, torch.int32, torch.int64)


def _blocks(size):
    return -(-size // X.BLOCK)


def _checked(name, tensor, shape, device, types=TYPES):
    """the tensor, dense: the library's calls take addresses and believe what they are told of the memory behind them"""
    if tensor.dtype in types and tensor.shape == shape and tensor.device == device and tensor.is_cuda:
        return tensor.contiguous()
    if tensor.dtype not in types:
        raise TypeError(f"{name}: {tensor.dtype} is none of {', '.join(str(t) for t in types)}")
    if tensor.shape != shape:
        raise ValueError(f"{name}: shape {tuple(tensor.shape)}, expected {tuple(shape)}")
    raise ValueError(f"{name}: on {tensor.device}, expected on {device if device.type == 'cuda' else 'the GPU'}")


def dense_ids(ids, experts):
    """ids as the sort reads them; what 32 bits cannot hold stays outside 0 .. experts-1 instead of losing its upper half"""
    if ids.dtype == torch.int64:
        ids = ids.clamp(-1, experts)
    return ids.to(torch.int32).contiguous()


class Quantized:
    """an 8-bit matrix with its scales; rows start on 16 bytes"""

    def __init__(self, rows, cols, scale_rows=None, batch=None, device="cuda"):
        lead = -(-cols // 16) * 16
        shape = () if batch is None else (batch,)
        self.q = torch.empty(*shape, rows, lead, dtype=torch.uint8, device=device)
        self.s = torch.empty(*shape, rows if scale_rows is None else scale_rows, _blocks(cols), device=device)

    def at(self):
        return self.q, self.q.stride(-2), self.s, self.s.stride(-2)

    def each(self):
        return self.q, self.q.stride(1), self.q.stride(0), self.s, self.s.stride(1), self.s.stride(0)


NONE = (None, 0, None, 0)


class Routes:
    """tokens sorted by expert"""

    def __init__(self, ids, experts, device=None):
        if ids.dim() != 2:
            raise ValueError(f"ids: shape {tuple(ids.shape)}, expected tokens x fan")
        ids = _checked("ids", ids, ids.shape, device or ids.device, INDEX_TYPES)
        self.tokens, self.fan = ids.shape
        self.experts, self.rows = experts, ids.numel()
        new = lambda n: torch.empty(n, dtype=torch.int32, device=ids.device)  # noqa: E731
        self.offsets, self.position, self.source = new(experts + 1), new(self.rows), new(self.rows)
        need = X.mg_expert_sort_workspace_bytes(self.tokens, self.fan, experts)
        workspace = torch.empty(need, dtype=torch.uint8, device=ids.device) if need else None
        X.mg_expert_sort(self.tokens, self.fan, experts, dense_ids(ids, experts), self.offsets, self.position, self.source, workspace)


class Experts:
    """the products of all experts with one matrix each: weights experts x n x k"""

    def __init__(self, weights):
        if weights.dim() != 3:
            raise ValueError(f"weights: shape {tuple(weights.shape)}, expected experts x n x k")
        self.weights = _checked("weights", weights, weights.shape, weights.device)
        self.experts, self.n, self.k = weights.shape
        self.w = Quantized(self.n, self.k, _blocks(self.n), self.experts, weights.device)
        self.turned = Quantized(self.k, self.n, _blocks(self.k), self.experts, weights.device)
        self.quantize()

    def quantize(self):
        """after a change of the weights: both forms that the products read, in one pass"""
        w = _checked("weights", self.weights, (self.experts, self.n, self.k), self.w.q.device)
        X.mg_block_quantize_batched(TYPES[w.dtype], X.MG_BLOCK_SQUARE, self.experts, self.n, self.k, w, self.k, self.n * self.k, *self.w.each(), *self.turned.each())

    def _rows(self, name, tensor, routes, of_tokens, cols):
        if routes.experts != self.experts:
            raise ValueError(f"routes to {routes.experts} experts, weights of {self.experts}")
        if routes.offsets.device != self.w.q.device:
            raise ValueError(f"routes on {routes.offsets.device}, weights on {self.w.q.device}")
        return _checked(name, tensor, (routes.tokens if of_tokens else routes.rows, cols), self.w.q.device)

    def _product(self, routes, a, source, fan, b, n, k, dtype):
        c = torch.empty(routes.rows, n, dtype=dtype, device=a.q.device)
        need = X.mg_block_gemm_grouped_workspace_bytes(self.experts, routes.rows, n, k)
        workspace = torch.empty(need, dtype=torch.uint8, device=a.q.device) if need else None
        X.mg_block_gemm_grouped(self.experts, routes.offsets, routes.rows, n, k, 1.0, X.MG_SCALES_POW2, *a.at(), source, fan, X.MG_BLOCK_SQUARE, *b.each(), 0.0,
                                TYPES[dtype], c, n, workspace)
        return c

    def forward(self, routes, x, of_tokens):
        """x: a row for each token (of_tokens: the products fetch every route's) or for each routed row"""
        return self._forward(routes, self._rows("x", x, routes, of_tokens, self.k), of_tokens)

    def _forward(self, routes, x, of_tokens):
        a = Quantized(x.shape[0], self.k, device=x.device)
        X.mg_block_quantize(TYPES[x.dtype], X.MG_BLOCK_ROW, x.shape[0], self.k, x, self.k, *a.at(), *NONE)
        return self._product(routes, a, routes.source if of_tokens else None, routes.fan if of_tokens else 1, self.w, self.n, self.k, x.dtype)

    def backward(self, routes, x, of_tokens, dy):
        """(gradient of the routed rows of x, gradient of the weights in FP32)"""
        x, dy = self._rows("x", x, routes, of_tokens, self.k), self._rows("dy", dy, routes, False, self.n)
        rows, columns = routes.rows, X.mg_grouped_columns(routes.rows, self.experts)
        d, d_turned, x_turned = (Quantized(*size, device=dy.device) for size in ((rows, self.n), (self.n, columns), (self.k, columns)))
        source, fan = (routes.source, routes.fan) if of_tokens else (None, 1)
        X.mg_block_quantize_grouped(TYPES[dy.dtype], self.experts, routes.offsets, rows, self.n, dy, self.n, None, 1, *d.at(), *d_turned.at())
        X.mg_block_quantize_grouped(TYPES[x.dtype], self.experts, routes.offsets, rows, self.k, x, self.k, source, fan, *NONE, *x_turned.at())
        dx = self._product(routes, d, None, 1, self.turned, self.k, self.n, dy.dtype)
        dw = torch.empty(self.experts, self.n, self.k, device=dy.device)
        need = X.mg_block_gemm_grouped_sum_workspace_bytes(self.experts, rows, self.n, self.k)
        workspace = torch.empty(need, dtype=torch.uint8, device=dy.device) if need else None
        X.mg_block_gemm_grouped_sum(self.experts, routes.offsets, rows, self.n, self.k, 1.0, X.MG_SCALES_POW2, *d_turned.at(), *x_turned.at(), 0.0, X.MG_F32, dw, self.k,
                                    self.n * self.k, workspace)
        return dx, dw


class ExpertLayer:
    """weights: W1 experts x hidden x width, W2 experts x width x hidden, of one type.  Outside autograd: results carry no graph, `backward` gives the gradients."""

    def __init__(self, w1, w2):
        if w1.dim() != 3 or tuple(w2.shape) != (w1.shape[0], w1.shape[2], w1.shape[1]):
            raise ValueError(f"weights: shapes {tuple(w1.shape)} and {tuple(w2.shape)}, expected experts x hidden x width and experts x width x hidden")
        self.up, self.down = Experts(w1), Experts(w2)
        self.width = w1.shape[2]
        self.kept = None

    def forward(self, x, ids, gates, keep=True):
        """x: tokens x width; ids: tokens x fan (negative: dropped); gates: tokens x fan (numbers of 16 bits are widened to the FP32 that the kernels read);
        keep: hold on to what `backward` reads, in place of an earlier call's (without: to nothing, as for tokens that are served)"""
        device = self.up.w.q.device
        x = _checked("x", x, (*ids.shape[:1], self.width), device)
        gates = _checked("gates", gates, ids.shape, device).float()
        routes = Routes(ids, self.up.experts, device)
        h = self.up._forward(routes, x, of_tokens=True)
        a = torch.relu(h).square_()
        rows = self.down._forward(routes, a, of_tokens=False)
        y = torch.empty_like(x)
        X.mg_expert_combine(TYPES[x.dtype], routes.tokens, routes.fan, self.width, rows, self.width, routes.position, gates, y, self.width)
        self.kept = (routes, x, gates, h, a, rows) if keep else None
        return y

    def backward(self, dy):
        """gradients (x, gates, W1, W2) of the last forward pass; dy of x's type, the gradients of gates and weights in FP32"""
        if self.kept is None:
            raise RuntimeError("backward without a forward pass that kept its activations")
        routes, x, gates, h, a, rows = self.kept
        dy = _checked("dy", dy, x.shape, x.device, (x.dtype,))
        code = TYPES[dy.dtype]
        d_rows, d_gates = torch.empty_like(rows), torch.empty_like(gates)
        X.mg_expert_combine_grad(code, routes.tokens, routes.fan, self.width, dy, self.width, rows, self.width, routes.position, gates, d_rows, self.width, d_gates)
        da, dw2 = self.down.backward(routes, a, False, d_rows)
        dh = da * (2 * torch.relu(h))
        d_routed, dw1 = self.up.backward(routes, x, True, dh)
        dx = torch.empty_like(x)
        X.mg_expert_combine(code, routes.tokens, routes.fan, self.width, d_routed, self.width, routes.position, None, dx, self.width)
        return dx, d_gates, dw1, dw2


def main(tokens=4096, width=1024, hidden=2048, experts=16, fan=2, steps=20, dtype=torch.bfloat16):
    gen = torch.Generator(device="cuda").manual_seed(1)
    normal = lambda *shape: torch.randn(*shape, device="cuda", generator=gen)  # noqa: E731
    make = lambda: ((normal(experts, hidden, width) * width ** -0.5).to(dtype), (normal(experts, width, hidden) * hidden ** -0.5).to(dtype))  # noqa: E731
    teacher, layer = ExpertLayer(*make()), ExpertLayer(*make())
    ids = torch.topk(normal(tokens, experts), fan).indices
    gates = torch.softmax(normal(tokens, fan), 1)
    x = normal(tokens, width).to(dtype)
    target = teacher.forward(x, ids, gates, keep=False)
    begin, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    for step in range(steps):
        begin.record()
        y = layer.forward(x, ids, gates)
        dy = y - target
        _, _, dw1, dw2 = layer.backward(dy)
        for part, grad in ((layer.up, dw1), (layer.down, dw2)):
            rms = grad.square().mean((1, 2), keepdim=True).sqrt() + 1e-20
            part.weights.sub_((0.02 * part.k ** -0.5 * grad / rms).to(dtype))
            part.quantize()
        end.record()
        torch.cuda.synchronize()
        loss = float(dy.float().square().mean())
        print(f"step {step:3d}  loss {loss:.4f}  {begin.elapsed_time(end):.3f} ms", flush=True)
    one = layer.forward(x[:1], ids[:1], gates[:1], keep=False)         # a token that is being generated
    print(f"one token: {float((one - target[:1]).float().square().mean()):.4f}")


if __name__ == "__main__":
    main(*(int(a) for a in sys.argv[1:6]))

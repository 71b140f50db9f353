"""Dense layers of a language model on the entry points of layers.py: a gated feed-forward block, the loss over a vocabulary, clipping of gradients.

    block  y = Wd (act(Wg x) * Wu x)          loss[t] = -log softmax(W x[t])[target[t]]          clip  g <- g min(1, max_norm / |all g|)

    python -m paper_1705_05249_amd.dense_layers [tokens] [width] [hidden] [vocab]

trains a block under a loss on tokens that another model has labelled, with clipped gradients, and prints loss, norm and the time of a step.  In the
manner of expert_layer.py: outside autograd, `backward` gives the gradients; PyTorch holds the memory and makes the update, everything else runs in the
library's kernels.  All buffers are allocated by the layers, on their weights' device, none by the library; the calls go to torch's current stream, so
that device has to be the current one.  Views are used where they are; 16-bit ones whose rows lie off 16 bytes (wide[:, 1:4097]) make large calls 2.7 to 4.5
times as long as their .contiguous() does.  What `forward` keeps (its inputs as they are, not copies of them) belongs to its stream: `backward` goes to the same one.
"""
import sys

import torch

from . import layers as L

TYPES = {torch.float32: L.MG_F32, torch.float16: L.MG_F16, torch.bfloat16: L.MG_BF16}
ACTIVATIONS = {"silu": L.MG_ACT_SILU, "gelu": L.MG_ACT_GELU, "gelu_tanh": L.MG_ACT_GELU_TANH, "relu2": L.MG_ACT_RELU2}


def _check_current(name, device):
    if device.index != torch.cuda.current_device():
        raise ValueError(f"{name}: on {device}, but the current device is cuda:{torch.cuda.current_device()}")


def _checked(name, tensor, shape, device, types):
    """the tensor with dense rows: the library's calls take addresses and believe what they are told of the memory behind them"""
    if tensor.dtype not in types:
        raise TypeError(f"{name}: {tensor.dtype} is none of {', '.join(str(t) for t in types)}")
    if tensor.shape != shape:
        raise ValueError(f"{name}: shape {tuple(tensor.shape)}, expected {tuple(shape)}")
    if tensor.device != device or not tensor.is_cuda:
        raise ValueError(f"{name}: on {tensor.device}, expected on {device if device.type == 'cuda' else 'the GPU'}")
    _check_current(name, device)
    tensor = tensor.detach()
    if tensor.dim() == 2 and tensor.numel() and (tensor.stride(1) != 1 or tensor.stride(0) < tensor.shape[1]):
        return tensor.contiguous()
    return tensor if tensor.dim() == 2 else tensor.contiguous()


def _at(matrix):
    """address and leading dimension"""
    return matrix, max(matrix.stride(0), matrix.shape[1], 1)


def _scratch(size, device):
    return torch.empty(size, dtype=torch.uint8, device=device) if size else None


class GatedBlock:
    """weights: gate and up, hidden x width, and down, width x hidden, of one type (views with dense rows are used where they are, so that an update of them is seen; of others
    a copy is made once)"""

    def __init__(self, gate, up, down, activation="silu"):
        if gate.dim() != 2 or up.shape != gate.shape or tuple(down.shape) != (gate.shape[1], gate.shape[0]):
            raise ValueError(f"weights: shapes {tuple(gate.shape)}, {tuple(up.shape)} and {tuple(down.shape)}, expected hidden x width twice and width x hidden")
        if activation not in ACTIVATIONS:
            raise ValueError(f"activation {activation!r} is none of {', '.join(ACTIVATIONS)}")
        self.hidden, self.width = gate.shape
        self.device, self.dtype = gate.device, gate.dtype
        self.gate, self.up, self.down = (_checked(name, w, w.shape, self.device, (self.dtype,) if name != "gate" else TYPES)
                                         for name, w in (("gate", gate), ("up", up), ("down", down)))
        self.activation = ACTIVATIONS[activation]
        self.kept = None

    def _size(self, tokens):
        return TYPES[self.dtype], tokens, self.width, self.hidden

    def forward(self, x, keep=True):
        """x: tokens x width of the weights' type; keep: hold on to what `backward` reads, in place of an earlier call's"""
        x = _checked("x", x, (x.shape[0], self.width), self.device, (self.dtype,))
        size = self._size(x.shape[0])
        y = torch.empty(x.shape, dtype=x.dtype, device=x.device)
        kept = _scratch(L.mg_gated_kept_bytes(*size), x.device) if keep else None
        workspace = _scratch(L.mg_gated_forward_workspace_bytes(*size), x.device)
        L.mg_gated_forward(size[0], self.activation, *size[1:], *_at(x), *_at(self.gate), *_at(self.up), *_at(self.down), *_at(y), kept, workspace)
        self.kept = (x, kept) if keep else None
        return y

    def backward(self, dy):
        """gradients (x, gate, up, down) of the last forward pass that kept its activations, of the weights' type"""
        if self.kept is None:
            raise RuntimeError("backward without a forward pass that kept its activations")
        x, kept = self.kept
        dy = _checked("dy", dy, x.shape, self.device, (self.dtype,))
        size = self._size(x.shape[0])
        grads = [torch.empty(t.shape, dtype=t.dtype, device=t.device) for t in (x, self.gate, self.up, self.down)]
        workspace = _scratch(L.mg_gated_backward_workspace_bytes(*size), x.device)
        L.mg_gated_backward(size[0], self.activation, *size[1:], *_at(x), *_at(self.gate), *_at(self.up), *_at(self.down), *_at(dy), kept,
                            *(v for g in grads for v in _at(g)), workspace)
        return tuple(grads)


class VocabLoss:
    """the last projection, weights vocab x width, and the cross entropy behind it"""

    def __init__(self, weights):
        if weights.dim() != 2:
            raise ValueError(f"weights: shape {tuple(weights.shape)}, expected vocab x width")
        self.weights = _checked("weights", weights, weights.shape, weights.device, TYPES)
        self.vocab, self.width = weights.shape
        self.kept = None

    def forward(self, x, targets, keep=True):
        """losses of the tokens in FP32, 0 where the target is outside the vocabulary (an ignored token); x: tokens x width, targets: 64-bit integers"""
        w = self.weights
        x = _checked("x", x, (x.shape[0], self.width), w.device, (w.dtype,))
        targets = _checked("targets", targets, x.shape[:1], w.device, (torch.int64,))
        size = TYPES[w.dtype], x.shape[0], self.width, self.vocab
        loss, lse = (torch.empty(x.shape[0], dtype=torch.float32, device=x.device) for _ in range(2))
        L.mg_vocab_loss(*size, *_at(x), *_at(w), targets, loss, lse, _scratch(L.mg_vocab_loss_workspace_bytes(*size), x.device))
        self.kept = (x, targets, lse) if keep else None
        return loss

    def backward(self, token_weights=None):
        """gradients (x, weights) of the sum of the losses, each times its token's weight (FP32; without: 1)"""
        if self.kept is None:
            raise RuntimeError("backward without a forward pass that kept its inputs")
        w = self.weights
        _check_current("weights", w.device)
        x, targets, lse = self.kept
        if token_weights is not None:
            token_weights = _checked("token_weights", token_weights, x.shape[:1], w.device, (torch.float32,))
        size = TYPES[w.dtype], x.shape[0], self.width, self.vocab
        dx, dw = (torch.empty(t.shape, dtype=t.dtype, device=t.device) for t in (x, w))
        L.mg_vocab_loss_grad(*size, *_at(x), *_at(w), targets, lse, token_weights, *_at(dx), *_at(dw), _scratch(L.mg_vocab_loss_grad_workspace_bytes(*size), x.device))
        return dx, dw


class Gradients:
    """dense tensors whose norm is taken together; listed once, for as long as they stay where they are.  Every call has a result and a workspace of its own; `value` is the last one's
    result"""

    def __init__(self, tensors):
        self.tensors = list(tensors)
        for i, t in enumerate(self.tensors):
            if t.dtype not in TYPES:
                raise TypeError(f"tensor {i}: {t.dtype} is none of {', '.join(str(k) for k in TYPES)}")
            if not t.is_cuda or t.device != self.tensors[0].device:
                raise ValueError(f"tensor {i}: on {t.device}, expected on {self.tensors[0].device if self.tensors[0].is_cuda else 'the GPU'}")
            _check_current(f"tensor {i}", t.device)
            if not t.is_contiguous():
                raise ValueError(f"tensor {i}: not dense")
        # (scaled in place, a number that is listed twice would be scaled twice)
        places = sorted((t.data_ptr(), t.data_ptr() + t.numel() * t.element_size(), i) for i, t in enumerate(self.tensors) if t.numel())
        for (_, end, i), (start, _, j) in zip(places, places[1:]):
            if start < end:
                raise ValueError(f"tensors {min(i, j)} and {max(i, j)} share memory")
        self.count = len(self.tensors)
        self.device = self.tensors[0].device if self.tensors else torch.device("cuda", torch.cuda.current_device())
        self.types = torch.tensor([TYPES[t.dtype] for t in self.tensors], dtype=torch.int32, device="cpu")
        self.addresses = torch.tensor([t.data_ptr() for t in self.tensors], dtype=torch.int64, device="cpu")
        self.sizes = torch.tensor([t.numel() for t in self.tensors], dtype=torch.int64, device="cpu")
        self.value = self._result()

    def _result(self):
        return torch.empty(1, dtype=torch.float32, device=self.device)

    def _workspace(self):
        return _scratch(L.mg_gradient_workspace_bytes(self.count), self.device)

    def norm(self):
        """the norm of all of them, FP32, one element"""
        _check_current("tensors", self.device)
        value = self.value = self._result()
        L.mg_gradient_norm(self.count, self.types, self.addresses, self.sizes, value, self._workspace())
        return value

    def clip(self, max_norm):
        """scales them in place where their norm is larger; the norm in front of that"""
        _check_current("tensors", self.device)
        value = self.value = self._result()
        L.mg_gradient_clip(self.count, self.types, self.addresses, None, self.sizes, float(max_norm), value, self._workspace())
        return value


def train_step(block, head, x, targets, max_norm):
    """(losses, norm of all gradients, gradients of gate, up, down and head, clipped) of x + block(x) under the head's loss, a mean over the tokens that count"""
    y = x + block.forward(x)
    loss = head.forward(y, targets)
    counted = ((targets >= 0) & (targets < head.vocab)).sum().clamp(min=1)
    dy, dhead = head.backward(torch.ones_like(loss) / counted)
    _, dgate, dup, ddown = block.backward(dy)
    grads = [dgate, dup, ddown, dhead]
    return loss, Gradients(grads).clip(max_norm), grads


def main(tokens=4096, width=1024, hidden=2816, vocab=8192, steps=20, dtype=torch.bfloat16):
    gen = torch.Generator(device="cuda").manual_seed(1)
    normal = lambda rows, cols: (torch.randn(rows, cols, device="cuda", generator=gen) * cols ** -0.5).to(dtype)  # noqa: E731
    make = lambda: (GatedBlock(normal(hidden, width), normal(hidden, width), normal(width, hidden)), VocabLoss(normal(vocab, width)))  # noqa: E731
    teacher, model = make(), make()
    x = torch.randn(tokens, width, device="cuda", generator=gen).to(dtype)
    targets = ((x + teacher[0].forward(x, keep=False)).float() @ teacher[1].weights.float().T).argmax(1)
    begin, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    for step in range(steps):
        begin.record()
        loss, norm, grads = train_step(*model, x, targets, max_norm=1.0)
        for w, g in zip((model[0].gate, model[0].up, model[0].down, model[1].weights), grads):
            w.sub_((2.0 * g.float()).to(dtype))
        end.record()
        torch.cuda.synchronize()
        print(f"step {step:3d}  loss {float(loss.mean()):.4f}  norm {float(norm):.3f}  {begin.elapsed_time(end):.3f} ms", flush=True)


if __name__ == "__main__":
    main(*(int(a) for a in sys.argv[1:5]))

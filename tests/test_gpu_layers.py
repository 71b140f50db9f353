"""Gated blocks, the loss over a vocabulary and clipping on the GPU against 64 bits (layer_reference.py), within bounds element by element."""
import functools
import math
import threading

import pytest
import torch

from paper_1705_05249_amd import dense_layers as D, layers as L
from tests import layer_reference as R

pytestmark = pytest.mark.gpu

KINDS = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
CODES = {torch.float32: L.MG_F32, torch.float16: L.MG_F16, torch.bfloat16: L.MG_BF16}
MARK = -77.0                                # what memory outside the results holds


def say(*what):
    print(*what, flush=True)


def normal(seed, *shape, sigma=1.0):
    return torch.randn(*shape, generator=torch.Generator().manual_seed(seed)) * sigma


class Held:
    """a matrix on the GPU inside a larger allocation: `lead` elements in front of it and rows `ld` apart, everything else MARK (or NaN around an operand)"""

    def __init__(self, x, lead=0, extra=0, around=math.nan):
        rows, cols = x.shape
        self.ld = max(cols + extra, 1)
        self.all = torch.full((lead + rows * self.ld + 64,), around, dtype=x.dtype)
        view = self.all[lead:lead + rows * self.ld].view(rows, self.ld)[:, :cols]
        view.copy_(x)
        self.mask = torch.ones(self.all.shape, dtype=torch.bool)
        self.mask[lead:lead + rows * self.ld].view(rows, self.ld)[:, :cols] = False
        self.host, self.all = self.all.clone(), self.all.cuda()
        self.x = self.all[lead:lead + rows * self.ld].view(rows, self.ld)[:, :cols]

    def at(self):
        return self.x.data_ptr(), self.ld

    def untouched(self):
        bits = torch.int32 if self.all.dtype == torch.float32 else torch.int16
        return torch.equal(self.all.cpu().view(bits)[self.mask], self.host.view(bits)[self.mask])


def result(rows, cols, dtype, lead=0, extra=0):
    return Held(torch.full((rows, cols), MARK, dtype=dtype), lead, extra, around=MARK)


def scratch(size):
    """a workspace of exactly that size, full of NaN, with a guard behind it"""
    held = torch.full((size + 4096,), 255, dtype=torch.uint8, device="cuda")
    return held, held[:size]


# (tokens, width, hidden): one of everything, ends inside pieces of 8, 16, 64 and tiles of 64, 128, 256, sums of one and of many pieces
BLOCKS = [(1, 1, 1), (1, 8, 16), (2, 64, 15), (3, 200, 129), (17, 33, 100), (64, 64, 64), (65, 136, 72), (130, 257, 65), (300, 72, 264), (257, 520, 136), (1, 520, 600), (9, 1000, 31),
          (33, 96, 300), (5, 2056, 40), (150, 2008, 500)]


def run_block(case, act, dtype, lead=0, extra=0, keep=True, backward=True, wanted=(True,) * 4, room=0):
    """lead, extra: of every matrix, or one for each of X, WG, WU, WD, Y, dY and the four results; room: bytes of workspace beyond what the queries answer"""
    tokens, width, hidden = case
    leads, extras = (v if isinstance(v, tuple) else (v,) * 10 for v in (lead, extra))
    code, kind = CODES[dtype], D.ACTIVATIONS[act]
    x, wg, wu, wd, dy = (t.to(dtype) for t in (normal(1, tokens, width), normal(2, hidden, width, sigma=width ** -0.5), normal(3, hidden, width, sigma=width ** -0.5),
                                                normal(4, width, hidden, sigma=hidden ** -0.5), normal(5, tokens, width)))
    where = "cuda" if tokens * width * hidden > 1 << 24 else "cpu"
    want = R.block(*(t.to(where) for t in (x, wg, wu, wd)), act, dtype, dy.to(where))
    held = [Held(t, *at) for t, *at in zip((x, wg, wu, wd), leads, extras)]
    arguments = [v for h in held for v in h.at()]
    y = result(tokens, width, dtype, leads[4], extras[4])
    kept_all, kept = scratch(L.mg_gated_kept_bytes(code, *case)) if keep else (None, None)
    ws_all, ws = scratch(L.mg_gated_forward_workspace_bytes(code, *case) + room)
    L.mg_gated_forward(code, kind, *case, *arguments, *y.at(), kept, ws)
    torch.cuda.synchronize()
    R.check(y.x, want["y"], "y")
    assert y.untouched() and bool((ws_all[len(ws):] == 255).all())
    assert kept_all is None or bool((kept_all[len(kept):] == 255).all())
    if not backward:
        return
    before = kept.clone()
    d = Held(dy, leads[5], extras[5])
    shapes = (tokens, width), (hidden, width), (hidden, width), (width, hidden)
    outs = [result(*shape, dtype, *at) if on else None for on, shape, *at in zip(wanted, shapes, leads[6:], extras[6:])]
    ws_all, ws = scratch(L.mg_gated_backward_workspace_bytes(code, *case) + room)
    L.mg_gated_backward(code, kind, *case, *arguments, *d.at(), kept, *(v for o in outs for v in (o.at() if o else (None, 0))), ws)
    torch.cuda.synchronize()
    for name, o in zip(("dx", "dwg", "dwu", "dwd"), outs):
        if o is not None:
            R.check(o.x, want[name], name)
            assert o.untouched(), name
    assert torch.equal(before, kept) and bool((ws_all[len(ws):] == 255).all())
    assert all(h.untouched() for h in held)


@pytest.mark.parametrize("dtype", KINDS)
@pytest.mark.parametrize("case", BLOCKS, ids=lambda c: "x".join(map(str, c)))
def test_block(case, dtype):
    say("block", case, dtype)
    run_block(case, R.ACTS[(sum(case) + len(dtype)) % 4], KINDS[dtype])


@pytest.mark.parametrize("act", R.ACTS)
@pytest.mark.parametrize("dtype", KINDS)
def test_activations(act, dtype):
    run_block((70, 80, 90), act, KINDS[dtype])


@pytest.mark.parametrize("dtype", KINDS)
@pytest.mark.parametrize("lead,extra", [(1, 0), (0, 1), (3, 5), (8, 8), (0, 24)])
@pytest.mark.parametrize("case", [(40, 72, 136), (33, 61, 75), (3, 264, 72)], ids=lambda c: "x".join(map(str, c)))
def test_block_of_parts_of_larger_matrices(case, lead, extra, dtype):
    run_block(case, "gelu_tanh", KINDS[dtype], lead, extra)


@pytest.mark.parametrize("dtype", KINDS)
@pytest.mark.parametrize("case", [(40, 72, 136), (300, 264, 520), (5, 136, 72)], ids=lambda c: "x".join(map(str, c)))
def test_blocks_whose_matrices_lie_differently(case, dtype):
    """every matrix has rows of its own distance, some of them off 16 bytes; with the workspace that the queries answer and with room for copies"""
    for lead, extra in ((0, (8, 24, 16, 40, 64, 32, 72, 80, 8, 48)), ((0, 3, 0, 8, 1, 0, 5, 0, 2, 0), (8, 24, 3, 40, 1, 32, 72, 5, 8, 48))):
        for room in (0, 1 << 22):
            run_block(case, "silu", KINDS[dtype], lead, extra, room=room)


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
def test_large_blocks_whose_matrices_lie_differently(dtype):
    """gate and up weights at different distances, on every tile that reads both in one sum"""
    for case in ((1000, 1000, 2000), (2100, 4000, 520), (4000, 1500, 700), (1500, 2000, 1000)):
        run_block(case, "gelu", KINDS[dtype], 0, (8, 24, 16, 40, 64, 32, 72, 80, 8, 48))


@pytest.mark.parametrize("dtype,ld", [("bf16", 1 << 20), ("f16", (1 << 21) + 8), ("bf16", (1 << 20) + 1), ("f32", 1 << 20)])
def test_rows_far_apart(dtype, ld):
    """operands and results whose last rows are more than 2^32 bytes behind the first"""
    kind = KINDS[dtype]
    tokens, width, hidden, code = 2100, 2064, 2072, CODES[kind]
    assert min(tokens, width, hidden) * ld * 2 > 1 << 32

    def far(x):
        room = torch.empty(x.shape[0] * ld, dtype=kind, device="cuda").view(-1, ld)[:, :x.shape[1]]
        room.copy_(x)
        return room
    data = [normal(i, r, c, sigma=1.0 if i in (1, 5) else c ** -0.5).to(kind) for i, (r, c) in enumerate(((tokens, width), (hidden, width), (hidden, width), (width, hidden), (tokens, width)), 1)]
    want = R.block(*(t.cuda() for t in data[:4]), "silu", kind, data[4].cuda())
    x, wg, wu, wd, dy = (far(t) for t in data)
    operands = [v for t in (x, wg, wu, wd) for v in (t.data_ptr(), ld)]
    zeros = lambda rows, cols: far(torch.zeros(rows, cols, dtype=kind))  # noqa: E731
    y = zeros(tokens, width)
    size = code, tokens, width, hidden
    kept = scratch(L.mg_gated_kept_bytes(*size))[1]
    L.mg_gated_forward(code, L.MG_ACT_SILU, *size[1:], *operands, y, ld, kept, scratch(L.mg_gated_forward_workspace_bytes(*size))[1])
    R.check(y, want["y"], "y")
    outs = [zeros(*t.shape) for t in (x, wg, wu, wd)]
    L.mg_gated_backward(code, L.MG_ACT_SILU, *size[1:], *operands, dy, ld, kept, *(v for o in outs for v in (o, ld)), scratch(L.mg_gated_backward_workspace_bytes(*size))[1])
    for name, o in zip(("dx", "dwg", "dwu", "dwd"), outs):
        R.check(o, want[name], name)
    del want
    targets = torch.randint(-1, hidden, (tokens,), generator=torch.Generator().manual_seed(3))
    want = R.loss(data[0].cuda(), data[1].cuda(), targets.cuda(), kind, None, gradient=True)
    loss, lse, target = torch.empty(tokens, device="cuda"), torch.empty(tokens, device="cuda"), targets.cuda()
    for o in outs[:2]:
        o.zero_()
    L.mg_vocab_loss(*size, *operands[:4], target, loss, lse, scratch(L.mg_vocab_loss_workspace_bytes(*size))[1])
    L.mg_vocab_loss_grad(*size, *operands[:4], target, lse, None, *(v for o in outs[:2] for v in (o, ld)), scratch(L.mg_vocab_loss_grad_workspace_bytes(*size))[1])
    for name, o in (("loss", loss), ("lse", lse), ("dx", outs[0]), ("dw", outs[1])):
        R.check(o, want[name], name)


@pytest.mark.parametrize("dtype", KINDS)
def test_infinities_stay_in_their_feature(dtype):
    """what a block keeps of one feature does not depend on what another one's is"""
    kind = KINDS[dtype]
    x, dy = (normal(1, 20, 16).abs() * 2).to(kind), normal(2, 20, 16, sigma=0.1).to(kind)
    weights = [normal(3, 40, 16).to(kind), normal(4, 40, 16).to(kind), normal(5, 16, 40).to(kind)]
    grads = []
    for largest in (False, True):
        if largest:
            weights[1][5] = torch.finfo(kind).max
        block = D.GatedBlock(*(w.cuda() for w in weights))
        block.forward(x.cuda())
        grads.append([g.cpu() for g in block.backward(dy.cuda())])
    others = torch.arange(40) != 5
    (_, gate, up, down), (_, gate2, up2, down2) = grads
    assert torch.equal(up, up2) and torch.equal(gate[others], gate2[others]) and torch.equal(down[:, others], down2[:, others])
    assert not bool(gate2[5].isfinite().all()) and bool(gate.isfinite().all())


@pytest.mark.parametrize("dtype", KINDS)
@pytest.mark.parametrize("case", [(1, 264, 72), (4, 1024, 520), (16, 64, 2048), (17, 513, 100), (48, 256, 256), (64, 1000, 1000), (100, 128, 64)], ids=lambda c: "x".join(map(str, c)))
def test_served_tokens(case, dtype):
    say("served", case, dtype)
    for lead, extra in ((0, 0), (1, 2)):
        run_block(case, "silu", KINDS[dtype], lead, extra, keep=False, backward=False)


@pytest.mark.parametrize("dtype", KINDS)
@pytest.mark.parametrize("wanted", [(True, False, False, False), (False, True, False, False), (False, False, True, False), (False, False, False, True), (False, True, True, False)])
def test_gradients_that_are_wanted(wanted, dtype):
    run_block((70, 72, 90), "gelu", KINDS[dtype], wanted=wanted)


# sizes at which one gradient alone is made on each of the tiles (tests/test_linear_plan.py)
ONE_GRADIENT = [(1500, 2000, 1000), (4000, 1500, 700), (2100, 4000, 520), (70, 72, 90), (1000, 1000, 2000), (700, 3000, 3000), (1200, 1000, 1000)]


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("case", ONE_GRADIENT, ids=lambda c: "x".join(map(str, c)))
def test_each_gradient_by_itself(case, dtype):
    say("one gradient", case, dtype)
    for wanted in ((True, False, False, False), (False, True, True, False), (False, False, False, True)):
        run_block(case, "silu", KINDS[dtype], wanted=wanted)


@pytest.mark.parametrize("dtype", KINDS)
def test_blocks_without_work(dtype):
    kind, code = KINDS[dtype], CODES[KINDS[dtype]]
    y = result(3, 5, kind, extra=2)
    w = torch.zeros(8, dtype=kind, device="cuda")
    L.mg_gated_forward(code, L.MG_ACT_SILU, 3, 5, 0, w, 5, w, 5, w, 5, w, 1, *y.at())
    assert not bool(y.x.any()) and y.untouched()
    outs = [result(*shape, kind, extra=1) for shape in ((0, 5), (4, 5), (4, 5), (5, 4))]
    L.mg_gated_backward(code, L.MG_ACT_SILU, 0, 5, 4, None, 5, w, 5, w, 5, w, 4, None, 5, None, *(v for o in outs for v in o.at()))
    torch.cuda.synchronize()
    assert all(not bool(o.x.any()) and o.untouched() for o in outs)


# (tokens, width, vocab)
LOSSES = [(1, 1, 1), (1, 8, 100), (2, 64, 65), (3, 33, 1000), (16, 256, 513), (17, 100, 64), (64, 72, 300), (70, 136, 1029), (130, 65, 200), (300, 264, 520), (257, 64, 257), (5, 1032, 4100), (150, 2008, 600)]


def run_loss(case, dtype, lead=0, extra=0, weights="each", ignored=0.3, wanted=(True, True), sigma=2.0, room=0):
    """lead, extra: of every matrix, or one for each of X, W, dX and dW"""
    tokens, width, vocab = case
    leads, extras = (v if isinstance(v, tuple) else (v,) * 4 for v in (lead, extra))
    code = CODES[dtype]
    x, w = normal(1, tokens, width).to(dtype), normal(2, vocab, width, sigma=sigma * width ** -0.5).to(dtype)
    gen = torch.Generator().manual_seed(3)
    targets = torch.randint(0, vocab, (tokens,), generator=gen)
    out = torch.rand(tokens, generator=gen) < ignored
    targets[out] = torch.tensor([-100, -1, vocab, 1 << 40, -(1 << 33)])[torch.arange(tokens) % 5][out]
    token_weights = {"each": torch.rand(tokens, generator=gen) * 2 - 0.5, "mean": torch.full((tokens,), 1.0 / 7001), "none": None, "large": torch.full((tokens,), 1024.0),
                     "zeros": torch.where(torch.arange(tokens) % 2 == 0, 0.0, 1.0)}[weights]
    where = "cuda" if tokens * width * vocab > 1 << 24 else "cpu"
    want = R.loss(x.to(where), w.to(where), targets.to(where), dtype, None if token_weights is None else token_weights.to(where), gradient=True)
    held = [Held(t, *at) for t, *at in zip((x, w), leads, extras)]
    arguments = [v for h in held for v in h.at()]
    target = targets.cuda()
    loss, lse = (result(1, tokens, torch.float32) for _ in range(2))
    ws_all, ws = scratch(L.mg_vocab_loss_workspace_bytes(code, *case) + room)
    L.mg_vocab_loss(code, *case, *arguments, target, loss.at()[0], lse.at()[0], ws)
    torch.cuda.synchronize()
    R.check(lse.x[0], want["lse"], "lse")
    R.check(loss.x[0], want["loss"], "loss")
    assert loss.untouched() and lse.untouched() and bool((ws_all[len(ws):] == 255).all())
    outs = [result(*shape, dtype, *at) if on else None for on, shape, *at in zip(wanted, ((tokens, width), (vocab, width)), leads[2:], extras[2:])]
    ws_all, ws = scratch(L.mg_vocab_loss_grad_workspace_bytes(code, *case) + room)
    L.mg_vocab_loss_grad(code, *case, *arguments, target, lse.at()[0], None if token_weights is None else token_weights.cuda(), *(v for o in outs for v in (o.at() if o else (None, 0))), ws)
    torch.cuda.synchronize()
    for name, o in zip(("dx", "dw"), outs):
        if o is not None:
            R.check(o.x, want[name], name)
            assert o.untouched(), name
    assert bool((ws_all[len(ws):] == 255).all()) and all(h.untouched() for h in held)
    counts = (targets >= 0) & (targets < vocab)
    if wanted[0]:
        assert not bool(outs[0].x.cpu()[~counts].any()) and not bool(loss.x[0].cpu()[~counts].any())       # ignored tokens: exactly nothing


@pytest.mark.parametrize("dtype", KINDS)
@pytest.mark.parametrize("case", LOSSES, ids=lambda c: "x".join(map(str, c)))
def test_loss(case, dtype):
    say("loss", case, dtype)
    run_loss(case, KINDS[dtype])


@pytest.mark.parametrize("dtype", KINDS)
@pytest.mark.parametrize("weights,ignored", [("mean", 0.0), ("none", 0.5), ("large", 0.1), ("zeros", 0.2), ("each", 1.0)])
def test_weights_of_tokens(weights, ignored, dtype):
    run_loss((40, 72, 333), KINDS[dtype], weights=weights, ignored=ignored)


@pytest.mark.parametrize("dtype", KINDS)
@pytest.mark.parametrize("lead,extra", [(1, 0), (0, 3), (8, 8)])
def test_loss_of_parts_of_larger_matrices(lead, extra, dtype):
    for case in ((40, 72, 136), (21, 45, 301)):
        run_loss(case, KINDS[dtype], lead, extra)


@pytest.mark.parametrize("dtype", KINDS)
@pytest.mark.parametrize("case", [(40, 72, 136), (250, 264, 520)], ids=lambda c: "x".join(map(str, c)))
def test_losses_whose_matrices_lie_differently(case, dtype):
    for lead, extra in ((0, (8, 24, 16, 40)), ((0, 3, 5, 0), (8, 5, 3, 40)), ((2, 0, 0, 1), (8, 16, 3, 40))):
        for room in (0, 1 << 22):
            run_loss(case, KINDS[dtype], lead, extra, room=room)


@pytest.mark.parametrize("dtype", KINDS)
def test_weights_of_all_sizes(dtype):
    """an infinite weight makes its own token's gradients no numbers and no other token's; tiny and huge ones are as exact as ordinary ones"""
    kind = KINDS[dtype]
    x, w, targets = normal(1, 40, 32).to(kind).cuda(), normal(2, 50, 32, sigma=0.2).to(kind).cuda(), (torch.arange(40) % 50).cuda()
    head = D.VocabLoss(w)
    head.forward(x, targets)
    ones = head.backward(torch.ones(40, device="cuda"))
    for scale in (2.0 ** -90, 2.0 ** 14):
        dx, dw = head.backward(torch.full((40,), scale, device="cuda"))
        if kind != torch.float16:                                    # (results are rounded to the type, whose range is what it is)
            assert all(torch.equal(a.double(), b.double() * scale) for a, b in zip((dx, dw), ones))
    some = torch.ones(40, device="cuda")
    some[7] = math.inf
    dx = head.backward(some)[0]
    others = torch.arange(40) != 7
    assert torch.equal(dx.cpu()[others], ones[0].cpu()[others]) and not bool(dx[7].isfinite().any())


@pytest.mark.parametrize("dtype", KINDS)
def test_weights_of_ignored_tokens(dtype):
    """they may be anything: what the gradient is rounded in goes by the tokens that count"""
    kind, vocab = KINDS[dtype], 90
    x, w = normal(1, 600, 40).to(kind).cuda(), normal(2, vocab, 40, sigma=0.2).to(kind).cuda()
    targets = torch.randint(0, vocab, (600,), generator=torch.Generator().manual_seed(3))
    ignored = torch.arange(600) % 3 == 1
    targets[ignored] = torch.tensor([-100, -1, vocab, 1 << 40, -(1 << 63)])[torch.arange(600) % 5][ignored]
    weights = torch.rand(600, generator=torch.Generator().manual_seed(4)) * 0.01
    head = D.VocabLoss(w)
    head.forward(x, targets.cuda())
    weights[ignored] = 0.0
    want = head.backward(weights.cuda())
    for other in (0.005, 1.0, 1e6, -1e30, 3e38, math.inf, -math.inf, math.nan):
        weights[ignored] = other
        got = head.backward(weights.cuda())
        assert all(torch.equal(a, b) for a, b in zip(got, want)), other
    # none counts: exactly nothing
    head.forward(x, torch.full((600,), -1, device="cuda"))
    assert not any(bool(t.any()) for t in head.backward(torch.full((600,), 1e6, device="cuda")))


@pytest.mark.parametrize("dtype", KINDS)
@pytest.mark.parametrize("wanted", [(True, False), (False, True)])
def test_gradients_of_the_loss_that_are_wanted(wanted, dtype):
    run_loss((40, 72, 333), KINDS[dtype], wanted=wanted)


@pytest.mark.parametrize("dtype", KINDS)
def test_sharp_logits(dtype):
    """far from each other: nearly all of the probability is one token's, or the largest logit is far above zero"""
    run_loss((33, 64, 400), KINDS[dtype], sigma=25.0, ignored=0.1)


@pytest.mark.parametrize("dtype", KINDS)
def test_losses_without_work(dtype):
    kind, code = KINDS[dtype], CODES[KINDS[dtype]]
    w = torch.zeros(64, dtype=kind, device="cuda")
    targets = torch.tensor([0, -1, 3], device="cuda")
    loss, lse = torch.full((3,), MARK, device="cuda"), torch.full((3,), MARK, device="cuda")
    ws = scratch(L.mg_vocab_loss_workspace_bytes(code, 3, 4, 0))[1]
    L.mg_vocab_loss(code, 3, 4, 0, w, 4, None, 4, targets, loss, lse, ws)
    assert loss.tolist() == [0.0] * 3 and lse.tolist() == [-math.inf] * 3
    ws = scratch(L.mg_vocab_loss_workspace_bytes(code, 3, 0, 7))[1]
    L.mg_vocab_loss(code, 3, 0, 7, None, 1, None, 1, targets, loss, lse, ws)                        # all logits zero
    assert torch.allclose(lse.cpu(), torch.full((3,), math.log(7.0))) and torch.allclose(loss.cpu(), torch.tensor([math.log(7.0), 0.0, math.log(7.0)]))
    dx, dw = result(3, 4, kind), result(6, 4, kind, extra=1)
    L.mg_vocab_loss_grad(code, 3, 4, 0, w, 4, None, 4, targets, lse, None, *dx.at(), None, 0)
    L.mg_vocab_loss_grad(code, 0, 4, 6, None, 4, w, 4, None, None, None, None, 0, *dw.at())
    assert not bool(dx.x.any()) and not bool(dw.x.any()) and dw.untouched() and dx.untouched()


@pytest.mark.parametrize("dtype", KINDS)
@pytest.mark.parametrize("tokens", [191, 192, 300, 5000])
def test_losses_without_width(tokens, dtype):
    """all logits are zero, on every kernel that many tokens take, wherever the empty rows start"""
    kind, code, targets = KINDS[dtype], CODES[KINDS[dtype]], torch.arange(tokens, device="cuda") % 8
    for vocab, ldx, ldw in ((7, 1, 1), (7, 8, 8), (2000, 3, 8)):
        loss, lse = (result(1, tokens, torch.float32) for _ in range(2))
        ws = scratch(L.mg_vocab_loss_workspace_bytes(code, tokens, 0, vocab))[1]
        L.mg_vocab_loss(code, tokens, 0, vocab, None, ldx, None, ldw, targets, loss.at()[0], lse.at()[0], ws)
        torch.cuda.synchronize()
        # a sum of `vocab` ones is exact, a logarithm off by a step
        assert bool(((lse.x[0].double() - math.log(vocab)).abs() <= R.STEP * math.log(vocab)).all()) and loss.untouched() and lse.untouched()
        assert torch.equal(loss.x[0], torch.where(targets < vocab, lse.x[0], 0.0))
    head = D.VocabLoss(torch.zeros(7, 0, dtype=kind, device="cuda"))
    loss = head.forward(torch.zeros(tokens, 0, dtype=kind, device="cuda"), targets)
    assert bool(((loss.double() - math.log(7)).abs() <= R.STEP * math.log(7))[targets < 7].all()) and not bool(loss[targets == 7].any())
    dx, dw = head.backward()
    assert dx.shape == (tokens, 0) and dw.shape == (7, 0)


def test_tokens_that_do_not_count_may_hold_anything():
    """infinities and NaN in ignored tokens and in tokens of weight zero stay where they are"""
    for kind in KINDS.values():
        x, w = normal(1, 20, 40), normal(2, 70, 40)
        x[3], x[5, 0], x[6, 1] = math.nan, math.inf, -math.inf
        targets = torch.randint(0, 70, (20,), generator=torch.Generator().manual_seed(1))
        targets[3] = -100
        weights = torch.ones(20)
        weights[5] = weights[6] = 0.0
        head = D.VocabLoss(w.to(kind).cuda())
        loss = head.forward(x.to(kind).cuda(), targets.cuda())
        dx, dw = head.backward(weights.cuda())
        fine = torch.ones(20, dtype=torch.bool)
        fine[[3, 5, 6]] = False
        assert bool(loss.cpu()[fine].isfinite().all()) and float(loss[3]) == 0.0
        assert bool(dx.cpu()[fine].isfinite().all()) and not bool(dx[[3, 5, 6]].any())
        # the same as without them
        x[[3, 5, 6]] = 0.0
        head.forward(x.to(kind).cuda(), targets.cuda())
        same_x, same_w = head.backward(weights.cuda())
        assert torch.equal(dx, same_x) and torch.equal(dw, same_w)


# sizes at which the large tiles are taken (tests/test_linear_plan.py says which by which product)
LARGE_BLOCKS = [(3999, 520, 4000), (4000, 4008, 520), (520, 4000, 2000), (3970, 515, 4001), (1500, 1032, 1000), (1000, 1000, 9992), (2500, 2600, 300), (2100, 520, 2500), (2100, 2048, 4100), (5500, 264, 5600)]


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("case", LARGE_BLOCKS, ids=lambda c: "x".join(map(str, c)))
def test_large_blocks(case, dtype):
    say("block", case, dtype)
    run_block(case, R.ACTS[sum(case) % 4], KINDS[dtype])


LARGE_LOSSES = [(4000, 520, 4000), (3970, 515, 4061), (1111, 1032, 2100), (2600, 264, 2600), (4000, 2000, 4000), (200, 512, 9000)]


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("case", LARGE_LOSSES, ids=lambda c: "x".join(map(str, c)))
def test_large_losses(case, dtype):
    say("loss", case, dtype)
    run_loss(case, KINDS[dtype])


@pytest.mark.parametrize("case,dtype", [((16500, 64, 16640), "bf16"), ((16500, 40, 16700), "f16"), ((5000, 64, 14000), "f32")])
def test_losses_in_pieces_of_the_vocabulary(case, dtype):
    """2^28 elements of dz (FP32: 2^26) are more than a piece"""
    assert case[0] * case[2] > (1 << 26 if dtype == "f32" else 1 << 28)
    run_loss(case, KINDS[dtype])


@pytest.mark.parametrize("dtype,tokens,vocab,pieces", [("bf16", 80000, 16640, 5), ("f16", 200000, 16701, 14), ("bf16", 160000, 10800, 8), ("f16", 100001, 10000, 4)])
def test_losses_in_more_pieces_than_slices(dtype, tokens, vocab, pieces):
    """every hundredth token counts, the others are ignored: dX of those and dW are what they alone give"""
    kind, code, width = KINDS[dtype], CODES[KINDS[dtype]], 72
    columns = (1 << 28) // tokens // 256 * 256
    assert -(-vocab // columns) == pieces
    x, w = normal(1, tokens, width).to(kind).cuda(), normal(2, vocab, width, sigma=2 * width ** -0.5).to(kind).cuda()
    some = torch.arange(7, tokens, 100, device="cuda")
    targets = torch.full((tokens,), -100, device="cuda")
    targets[some] = torch.randint(0, vocab, some.shape, generator=torch.Generator().manual_seed(3)).cuda()
    weights = torch.rand(tokens, generator=torch.Generator().manual_seed(4)).cuda() + 0.5
    want = R.loss(x[some], w, targets[some], kind, weights[some], gradient=True)
    lse = torch.zeros(tokens, device="cuda")
    lse[some] = want["lse"][0].float()
    size = code, tokens, width, vocab
    both = []
    for wanted in ((True, True), (True, False)):
        dx, dw = (result(*shape, kind) if on else None for on, shape in zip(wanted, ((tokens, width), (vocab, width))))
        ws_all, ws = scratch(L.mg_vocab_loss_grad_workspace_bytes(*size))
        L.mg_vocab_loss_grad(*size, x, width, w, width, targets, lse, weights, *dx.at(), *(dw.at() if dw else (None, 0)), ws)
        torch.cuda.synchronize()
        R.check(dx.x[some], want["dx"], "dx")
        others = torch.ones(tokens, dtype=torch.bool, device="cuda")
        others[some] = False
        assert not bool(dx.x[others].any()) and dx.untouched() and bool((ws_all[len(ws):] == 255).all())
        if dw:
            R.check(dw.x, want["dw"], "dw")
            assert dw.untouched()
        both.append(dx.x)
    assert torch.equal(*both)


# ---- clipping

def run_clip(sizes, kinds, max_norm, place, lead=0, scale=1.0):
    tensors = [Held((normal(i, 1, n) * scale).to(KINDS[k]), lead, around=MARK) for i, (n, k) in enumerate(zip(sizes, kinds))]
    before = [t.host[lead:lead + n].clone() for t, n in zip(tensors, sizes)]
    results = tensors if place == "in place" else [result(1, n, KINDS[k], lead) for n, k in zip(sizes, kinds)]
    total = math.sqrt(sum(float(b.double().square().sum()) for b in before))
    codes = torch.tensor([CODES[KINDS[k]] for k in kinds], dtype=torch.int32)
    at = lambda held: torch.tensor([h.at()[0] for h in held], dtype=torch.int64)  # noqa: E731
    norm = torch.full((1,), MARK, device="cuda")
    ws_all, ws = scratch(L.mg_gradient_workspace_bytes(len(sizes)))
    args = len(sizes), codes, at(tensors)
    L.mg_gradient_norm(*args, torch.tensor(sizes), norm, ws)
    assert abs(float(norm) - total) <= 2.0 ** -23 * total
    norm.fill_(MARK)
    ws_all.fill_(255)
    limit = max_norm * total if math.isfinite(max_norm) else max_norm
    limit = float(torch.tensor(limit))
    L.mg_gradient_clip(*args, None if place == "in place" else at(results), torch.tensor(sizes), limit, norm, ws)
    torch.cuda.synchronize()
    assert abs(float(norm) - total) <= 2.0 ** -23 * total and bool((ws_all[len(ws):] == 255).all())
    factor = torch.tensor(limit / total if limit < total else 1.0)
    for b, r, n, k in zip(before, results, sizes, kinds):
        got = r.x.cpu().view(-1)
        assert r.untouched()
        if limit >= total:
            assert torch.equal(got, b)
        elif n:
            # the factor is off by a step at most (the norm's 64-bit sum has another order), the product by half of one, the result by half a step of its type
            want = b.double() * factor.double()
            assert bool(((got.double() - want).abs() <= 2.0 ** -22 * want.abs() + R.HALF[KINDS[k]] * want.abs() * (1 + 2.0 ** -20) + R.TINY[KINDS[k]]).all())


@pytest.mark.parametrize("place", ["in place", "beside"])
@pytest.mark.parametrize("max_norm", [0.25, 1.5, math.inf])
@pytest.mark.parametrize("sizes", [(1,), (0, 3, 0), (7, 4096, 4097, 8192, 8193, 100), (100000, 1, 30000), tuple(range(130)), (300001,)], ids=lambda s: f"{len(s)}_{sum(s)}")
def test_clip(sizes, max_norm, place):
    kinds = [("f32", "f16", "bf16")[i % 3] for i in range(len(sizes))]
    say("clip", len(sizes), sum(sizes), max_norm, place)
    if sum(sizes) == 0:
        return
    run_clip(sizes, kinds, max_norm, place)


@pytest.mark.parametrize("kind", KINDS)
def test_clip_at_any_address(kind):
    run_clip((5000, 33, 70001), (kind,) * 3, 0.5, "beside", lead=1)
    run_clip((5000, 33, 70001), (kind,) * 3, 0.5, "in place", lead=3)


def test_squares_beyond_fp32():
    run_clip((5000, 600), ("f32", "bf16"), 0.5, "beside", scale=1e30)
    run_clip((5000, 600), ("f32", "bf16"), 0.5, "beside", scale=1e-30)


@pytest.mark.parametrize("kind", ["f32", "bf16"])
def test_norms_beyond_fp32(kind):
    """finite numbers whose norm is told as infinity: they stay as they are, in place and beside"""
    for numbers in ([3e38, 3e38, -1.0], [2.5e38] * 2 + [1e-3] * 5000):
        g = torch.tensor(numbers).to(KINDS[kind])
        held, beside = g.cuda(), torch.full(g.shape, MARK, dtype=g.dtype, device="cuda")
        assert bool(held.isfinite().all()) and float(held.double().norm()) > torch.finfo(torch.float32).max
        norm, ws = torch.empty(1, device="cuda"), scratch(L.mg_gradient_workspace_bytes(1))[1]
        args = 1, torch.tensor([CODES[g.dtype]], dtype=torch.int32), torch.tensor([held.data_ptr()])
        for results in (torch.tensor([beside.data_ptr()]), None):
            for limit in (1.0, 3e38, 0.0):
                norm.fill_(MARK)
                L.mg_gradient_clip(*args, results, torch.tensor([g.numel()]), limit, norm, ws)
                assert float(norm) == math.inf and torch.equal(held.cpu(), g) and (results is None or torch.equal(beside.cpu(), g)), (numbers[:3], limit)
    # just within the range: clipped, by a factor and with products that are off by half a step each
    g = torch.tensor([3e38, 1e38]).to(KINDS[kind]).cuda()
    assert math.isfinite(float(D.Gradients([g]).clip(2.0 ** 100))) and abs(float(g.double().norm()) / 2.0 ** 100 - 1.0) <= 2 * R.HALF[KINDS[kind]]


def test_limits_of_clipping():
    g = torch.tensor([3.0, 4.0, 0.0], device="cuda")
    grads = D.Gradients([g])
    assert float(grads.norm()) == 5.0
    assert float(grads.clip(5.0)) == 5.0 and g.tolist() == [3.0, 4.0, 0.0]              # no larger than the limit
    assert float(grads.clip(0.0)) == 5.0 and g.tolist() == [0.0, 0.0, 0.0]
    assert float(grads.clip(0.0)) == 0.0 and g.tolist() == [0.0, 0.0, 0.0]              # 0 / 0 is never formed
    for bad in (math.inf, -math.inf, math.nan):
        g.copy_(torch.tensor([1.0, bad, 2.0]))
        n = float(grads.clip(0.5))
        assert not math.isfinite(n) and math.isnan(n) == math.isnan(bad) and g[0] == 1.0 and g[2] == 2.0
    none = D.Gradients([])
    none.value.fill_(MARK)
    assert float(none.norm()) == 0.0
    none.value.fill_(MARK)
    assert float(none.clip(1.0)) == 0.0
    empty = D.Gradients([torch.empty(0, device="cuda")])
    assert float(empty.clip(1.0)) == 0.0


# ---- together, as a program uses them

def make(dtype, tokens=150, width=96, hidden=200, vocab=500, seed=10):
    block = D.GatedBlock(*(normal(seed + i, r, c, sigma=c ** -0.5).to(dtype).cuda() for i, (r, c) in enumerate(((hidden, width), (hidden, width), (width, hidden)))))
    head = D.VocabLoss(normal(seed + 3, vocab, width, sigma=width ** -0.5).to(dtype).cuda())
    x = normal(seed + 4, tokens, width).to(dtype).cuda()
    targets = torch.randint(-1, vocab, (tokens,), generator=torch.Generator().manual_seed(seed)).cuda()
    return block, head, x, targets


@functools.lru_cache(None)
def exact_step(dtype):
    block, head, x, targets = make(dtype)
    leaves = [t.double().cpu().requires_grad_() for t in (block.gate, block.up, block.down, head.weights)]
    xd, t = x.double().cpu(), targets.cpu()
    y = xd + (torch.nn.functional.silu(xd @ leaves[0].T) * (xd @ leaves[1].T)) @ leaves[2].T
    loss = torch.nn.functional.cross_entropy(y @ leaves[3].T, t.clamp(min=0), reduction="none") * (t >= 0)
    grads = torch.autograd.grad(loss.sum() / (t >= 0).sum(), leaves)
    norm = math.sqrt(sum(float(g.square().sum()) for g in grads))
    return loss.detach(), norm, [g * min(1.0, 0.05 / norm) for g in grads]


@pytest.mark.parametrize("dtype", KINDS)
def test_a_training_step(dtype):
    kind = KINDS[dtype]
    want_loss, want_norm, want = exact_step(kind)
    block, head, x, targets = make(kind)
    loss, norm, grads = D.train_step(block, head, x, targets, 0.05)
    # y and dy are rounded to the type between the block and the loss, H, dG, dU, dz and results once more: eight roundings of half a step at most, as parts of
    # norms; each logit's rounding of y moves a probability by up to |z| / sqrt(width) half steps beside them, which doubles it
    near = 16 * R.HALF[kind] + 1e-5
    assert float((loss.cpu().double() - want_loss).norm()) <= near * float(want_loss.norm())
    assert abs(float(norm) - want_norm) <= near * want_norm
    for g, w in zip(grads, want):
        assert float((g.cpu().double() - w).norm()) <= near * float(w.norm())


def graph_of(fn):
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        fn()
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = fn()
    return graph, out


@pytest.mark.parametrize("dtype", KINDS)
def test_a_captured_step_gives_what_an_eager_one_does(dtype):
    """bit for bit, on every replay, with the program's own work and new inputs between them; two graphs take turns"""
    block, head, x, targets = make(KINDS[dtype])
    xs = [x.clone(), make(KINDS[dtype], seed=20)[2]]

    def step(held):
        y = block.forward(held)
        loss = head.forward(y, targets)
        dy, dhead = head.backward()
        grads = [*block.backward(dy), dhead]
        return [loss, Clip(grads), y, *grads]

    def Clip(grads):
        g = D.Gradients(grads)
        lists.append(g)
        return g.clip(1.0)

    lists, eager = [], []
    for source in xs:
        eager.append([t.clone() for t in step(source)])
    held = [x.clone(), x.clone()]
    graphs = [graph_of(lambda h=h: step(h)) for h in held]
    for turn in range(4):
        for n, (graph, out) in enumerate(graphs):
            which = (turn + n) % 2
            held[n].copy_(xs[which])
            graph.replay()
            again = step(xs[1 - which])                       # the program's own work in between
            torch.cuda.synchronize()
            for k, (a, b) in enumerate(zip(out, eager[which])):
                assert torch.equal(a, b), (turn, n, k)
            for k, (a, b) in enumerate(zip(again, eager[1 - which])):
                assert torch.equal(a, b), (turn, n, k)


def test_calls_go_to_the_stream_they_are_given():
    block, head, x, targets = make(torch.bfloat16)
    want = [block.forward(x), head.forward(x, targets)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = [block.forward(x), head.forward(x, targets)]
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_layers_take_views_and_refuse_other_types():
    block, head, x, targets = make(torch.float16)
    wide = torch.zeros(x.shape[0], x.shape[1] + 5, dtype=x.dtype, device="cuda")
    wide[:, 2:-3] = x
    want = block.forward(x)
    assert torch.equal(block.forward(wide[:, 2:-3]), want) or float((block.forward(wide[:, 2:-3]).double() - want.double()).norm()) <= 2 ** -10 * float(want.double().norm())
    turned = x.T.contiguous().T
    assert torch.equal(block.forward(turned), want)
    with pytest.raises(TypeError):
        block.forward(x.float())
    with pytest.raises(ValueError):
        block.forward(x[:, :-1])
    with pytest.raises(TypeError):
        head.forward(x, targets.int())
    with pytest.raises(ValueError):
        head.forward(x, targets[:-1])
    with pytest.raises(ValueError):
        block.forward(x.cpu())
    with pytest.raises(ValueError):
        D.Gradients([x.T])
    block.forward(x, keep=False)
    with pytest.raises(RuntimeError):
        block.backward(x)


def test_two_streams_at_once():
    """calls that overlap, a workspace each, give what they give one after the other"""
    models = [make(torch.bfloat16, tokens=600, width=520, hidden=1000, vocab=3000, seed=s) for s in (30, 40)]
    want = [[t.clone() for t in D.train_step(block, head, x, targets, 0.05)[2]] for block, head, x, targets in models]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in models]
    got = [[], []]
    for _ in range(5):
        for n, (stream, model) in enumerate(zip(streams, models)):
            with torch.cuda.stream(stream):
                got[n].append(D.train_step(*model, 0.05)[2])
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for n in (0, 1) for grads in got[n] for a, b in zip(grads, want[n]))


def test_calls_from_several_threads():
    """the interpreter's lock is released in a call: every thread has a stream and workspaces of its own"""
    block, head, x, targets = make(torch.float16, tokens=300)
    want = [t.clone() for t in D.train_step(block, head, x, targets, 0.05)[2]]
    torch.cuda.synchronize()
    wrong = []

    def work():
        with torch.cuda.stream(torch.cuda.Stream()):
            model = D.GatedBlock(block.gate, block.up, block.down), D.VocabLoss(head.weights)
            for _ in range(10):
                grads = D.train_step(*model, x, targets, 0.05)[2]
            torch.cuda.current_stream().synchronize()
            wrong.extend(not torch.equal(a, b) for a, b in zip(grads, want))

    threads = [threading.Thread(target=work) for _ in range(4)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert len(wrong) == 16 and not any(wrong)


def test_other_default_types_and_devices():
    """buffers and tables have the types that the calls are told, whatever torch makes by default"""
    want = [t.clone() for t in D.train_step(*make(torch.bfloat16), 0.05)[2]]
    model = make(torch.bfloat16)
    torch.set_default_dtype(torch.bfloat16)
    torch.set_default_device("cuda")
    try:
        loss, norm, grads = D.train_step(*model, 0.05)
    finally:
        torch.set_default_dtype(torch.float32)
        torch.set_default_device("cpu")
    assert loss.dtype == norm.dtype == torch.float32 and all(torch.equal(a, b) for a, b in zip(grads, want))


def test_other_devices_are_refused(monkeypatch):
    """the calls would go to the current device's stream"""
    block, head, x, targets = make(torch.float16)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 1)
    with pytest.raises(ValueError, match="current device is cuda:1"):
        block.forward(x)
    with pytest.raises(ValueError, match="current device is cuda:1"):
        head.forward(x, targets)
    with pytest.raises(ValueError, match="current device is cuda:1"):
        D.Gradients([x])


def test_other_devices_are_refused_in_every_call(monkeypatch):
    """also by calls that take no tensor of their own"""
    block, head, x, targets = make(torch.float16)
    grads = D.Gradients([x])
    head.forward(x, targets)
    block.forward(x)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 1)
    for call in (head.backward, grads.norm, lambda: grads.clip(1.0), lambda: block.backward(x)):
        with pytest.raises(ValueError, match="current device is cuda:1"):
            call()


def test_norms_of_one_list_on_two_streams(monkeypatch):
    """every call has a result and a workspace of its own"""
    g = torch.tensor([3.0, 4.0], device="cuda")
    grads = D.Gradients([g])
    first = grads.norm()
    g.mul_(2.0)
    second = grads.clip(5.0)
    third = grads.norm()
    assert [float(t) for t in (first, second, third)] == [5.0, 10.0, 5.0] and g.tolist() == [3.0, 4.0]
    places = []
    for name in ("mg_gradient_norm", "mg_gradient_clip"):
        real = getattr(L, name)
        monkeypatch.setattr(L, name, lambda *a, real=real: places.append({t.data_ptr() for t in a[-2:]}) or real(*a))
    torch.cuda.synchronize()
    streams, norms = [torch.cuda.Stream() for _ in range(2)], []
    for stream in streams:
        with torch.cuda.stream(stream):
            norms.append(grads.norm())
            norms.append(grads.clip(100.0))
    torch.cuda.synchronize()
    assert [float(t) for t in norms] == [5.0] * 4
    assert not (places[0] | places[1]) & (places[2] | places[3])
    # two captured graphs and an eager call between their replays
    graphs = [graph_of(grads.norm) for _ in range(2)]
    for turn in range(4):
        for n, (graph, out) in enumerate(graphs):
            g.copy_(torch.tensor([3.0, 4.0], device="cuda") * (turn + n + 1))
            graph.replay()
            g.copy_(torch.tensor([6.0, 8.0], device="cuda"))
            assert float(grads.norm()) == 10.0 and float(out) == 5.0 * (turn + n + 1)


def test_memory_that_is_listed_twice():
    g = torch.ones(100, device="cuda")
    with pytest.raises(ValueError, match="0 and 1 share memory"):
        D.Gradients([g, g])
    with pytest.raises(ValueError, match="0 and 2 share memory"):
        D.Gradients([g[:51], torch.ones(3, device="cuda"), g[50:]])
    assert float(D.Gradients([g[:50], g[50:], g[7:7]]).norm()) == 10.0


def test_example_runs(capsys):
    D.main(tokens=96, width=64, hidden=80, vocab=200, steps=2)
    assert "step   1" in capsys.readouterr().out

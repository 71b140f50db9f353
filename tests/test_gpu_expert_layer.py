"""The layer of expert_layer.py against the same formulas in 64 bits, with the 8-bit roundings where the layer has them.

The layer's FP32 intermediates differ from the 64-bit ones by 1e-6 of them at most, so that now and then an element next to a tie is rounded to the
neighbouring 8-bit number: an eighth of itself, for at most one element in ten thousand (a tie's neighbourhood of 1e-6 among steps of 2^-4), which
changes a matrix's norm by less than 2^-3 * 1e-2; through two products and the activation's derivative 2^-8 of the norm at most."""
import numpy as np
import pytest
import torch

from paper_1705_05249_amd.expert_layer import ExpertLayer
from tests import expert_reference as R

pytestmark = pytest.mark.gpu


def rounded(x, square=False):
    return R.values(*R.quantize(x, square), square)


def reference(x, ids, gates, w1, w2, dy):
    tokens, fan = ids.shape
    y, dx = np.zeros_like(x), np.zeros_like(x)
    dgates, dw1, dw2 = np.zeros_like(gates), np.zeros_like(w1), np.zeros_like(w2)
    for e in range(w1.shape[0]):
        slots = [(t, j) for t in range(tokens) for j in range(fan) if ids[t, j] == e]
        if not slots:
            continue
        t, j = (np.array(s) for s in zip(*slots))
        q1, q2 = rounded(w1[e], True), rounded(w2[e], True)
        h = rounded(x[t]) @ q1.T
        a = np.maximum(h, 0) ** 2
        rows = rounded(a) @ q2.T
        g = gates[t, j]
        for i in range(len(t)):
            y[t[i]] += g[i] * rows[i]
        dgates[t, j] = (dy[t] * rows).sum(1)
        d_rows = g[:, None] * dy[t]
        da = rounded(d_rows) @ q2
        dw2[e] = rounded(d_rows.T) @ rounded(a.T).T
        dh = da * 2 * np.maximum(h, 0)
        d_routed = rounded(dh) @ q1
        dw1[e] = rounded(dh.T) @ rounded(x[t].T).T
        for i in range(len(t)):
            dx[t[i]] += d_routed[i]
    return y, dx, dgates, dw1, dw2


@pytest.mark.parametrize("tokens,width,hidden,experts,fan,dropped", ((37, 160, 200, 5, 2, 0.0), (1, 128, 256, 4, 3, 0.0), (150, 96, 131, 3, 1, 0.3), (20, 64, 64, 40, 2, 0.1)))
def test_forward_and_backward(tokens, width, hidden, experts, fan, dropped):
    rng = np.random.default_rng(tokens)
    ids = np.stack([rng.permutation(experts)[:fan] for _ in range(tokens)])
    ids[rng.random(ids.shape) < dropped] = -1
    x, dy = (rng.standard_normal((tokens, width)).astype(np.float32) for _ in range(2))
    gates = rng.uniform(0.1, 1, (tokens, fan)).astype(np.float32)
    w1 = (rng.standard_normal((experts, hidden, width)) * width ** -0.5).astype(np.float32)
    w2 = (rng.standard_normal((experts, width, hidden)) * hidden ** -0.5).astype(np.float32)
    layer = ExpertLayer(torch.tensor(w1).cuda(), torch.tensor(w2).cuda())
    y = layer.forward(torch.tensor(x).cuda(), torch.tensor(ids).cuda(), torch.tensor(gates).cuda())
    got = (y, *layer.backward(torch.tensor(dy).cuda()))
    want = reference(*(v.astype(np.float64) if v.dtype == np.float32 else v for v in (x, ids, gates, w1, w2, dy)))
    for name, g, r in zip(("y", "x", "gates", "W1", "W2"), got, want):
        g = g.double().cpu().numpy()
        assert np.linalg.norm(g - r) <= 2.0 ** -8 * np.linalg.norm(r), name
        if name in ("W1", "W2"):
            idle = [e for e in range(experts) if not (ids == e).any()]
            assert not g[idle].any()


def test_gradient_of_gates_against_differences():
    """the output is linear in the gates: a difference quotient is the gradient up to FP32's rounding"""
    rng = np.random.default_rng(0)
    tokens, width, hidden, experts, fan = 9, 64, 96, 4, 2
    ids = torch.tensor(np.stack([rng.permutation(experts)[:fan] for _ in range(tokens)])).cuda()
    x, dy = (torch.tensor(rng.standard_normal((tokens, width)), dtype=torch.float32).cuda() for _ in range(2))
    gates = torch.tensor(rng.uniform(0.2, 1, (tokens, fan)), dtype=torch.float32).cuda()
    layer = ExpertLayer(*(torch.tensor(rng.standard_normal(s) * s[2] ** -0.5, dtype=torch.float32).cuda() for s in ((experts, hidden, width), (experts, width, hidden))))
    layer.forward(x, ids, gates)
    _, d_gates, _, _ = layer.backward(dy)
    step = 2.0 ** -4
    for t, j in ((0, 0), (3, 1), (8, 0)):
        loss = []
        for sign in (1, -1):
            g = gates.clone()
            g[t, j] += sign * step
            loss.append(float((layer.forward(x, ids, g).double() * dy.double()).sum()))
        size = float(dy[t].abs().sum()) * 32
        assert abs((loss[0] - loss[1]) / (2 * step) - float(d_gates[t, j])) <= size * 2.0 ** -20


def test_views_as_arguments():
    """rows of a wider tensor, transposed weights and gates that are not dense give what their copies give"""
    rng = np.random.default_rng(3)
    tokens, width, hidden, experts, fan = 21, 96, 130, 3, 2
    new = lambda *shape: torch.tensor(rng.standard_normal(shape), dtype=torch.float32).cuda()  # noqa: E731
    ids = torch.tensor(rng.integers(0, experts, (tokens, fan))).cuda()
    x, dy, gates = new(tokens, width + 7)[:, 7:], new(width, tokens).T, new(fan, tokens).T
    w1, w2 = new(experts, width, hidden).transpose(1, 2), new(experts, hidden, width).transpose(1, 2)
    results = []
    for copy in (False, True):
        a = [t.contiguous() if copy else t for t in (x, dy, gates, w1, w2)]
        layer = ExpertLayer(a[3], a[4])
        results.append((layer.forward(a[0], ids, a[2]), *layer.backward(a[1])))
    assert all(torch.equal(p, q) for p, q in zip(*results))


def test_training_reaches_the_target(capsys):
    """the command: the loss falls by half in twenty steps"""
    from paper_1705_05249_amd import expert_layer
    expert_layer.main(tokens=512, width=256, hidden=256, experts=8, fan=2)
    lines = [line.split() for line in capsys.readouterr().out.splitlines() if line.startswith("step")]
    losses = [float(line[3]) for line in lines]
    assert len(losses) == 20 and losses[-1] < losses[0] / 2 and all(np.isfinite(losses))

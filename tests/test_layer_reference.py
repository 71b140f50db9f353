"""The 64-bit reference of the dense layers against differences of its own values and against torch's differentiation."""
import pytest
import torch

from tests import layer_reference as R


def normal(*shape, seed=0):
    return torch.randn(*shape, dtype=torch.float64, generator=torch.Generator().manual_seed(seed + sum(shape)))


@pytest.mark.parametrize("kind", R.ACTS)
def test_slopes_are_differences_of_the_activations(kind):
    g = normal(400) * 3
    a, slope, _ = R.act(g, kind)
    e = 1e-5
    assert torch.allclose((R.act(g + e, kind)[0] - R.act(g - e, kind)[0]) / (2 * e), slope, atol=1e-8, rtol=1e-8)
    bend = (R.act(g + e, kind)[1] - R.act(g - e, kind)[1]) / (2 * e)
    assert float(bend.abs().max()) <= 2.0 + 1e-6                # what the bounds take it to be
    torch_form = {"silu": torch.nn.functional.silu, "gelu": torch.nn.functional.gelu, "relu2": lambda v: torch.relu(v) ** 2,
                  "gelu_tanh": lambda v: torch.nn.functional.gelu(v, approximate="tanh")}[kind]
    assert torch.allclose(a, torch_form(g), atol=1e-12)


@pytest.mark.parametrize("kind", R.ACTS)
def test_gradients_of_a_block_are_differences(kind):
    x, wg, wu, wd, dy = normal(5, 4), normal(6, 4), normal(6, 4, seed=1), normal(4, 6), normal(5, 4, seed=2)
    got = R.block(x, wg, wu, wd, kind, torch.float32, dy)
    value = lambda *t: float((R.block(*t, kind, torch.float32)["y"][0] * dy).sum())  # noqa: E731
    inputs = [x, wg, wu, wd]
    for n, name in enumerate(("dx", "dwg", "dwu", "dwd")):
        for at in ((0, 0), (3, 2)):
            ends = []
            for e in (1e-5, -1e-5):
                moved = [t.clone() for t in inputs]
                moved[n][at] += e
                ends.append(value(*moved))
            assert abs((ends[0] - ends[1]) / 2e-5 - float(got[name][0][at])) < 1e-6 * (1 + abs(float(got[name][0][at]))), (name, at)


def test_gradients_of_the_loss_are_differences():
    x, w, targets, weights = normal(6, 5), normal(9, 5), torch.tensor([0, 8, -1, 3, 9, 3]), torch.tensor([1.0, 0.5, 2.0, 0.0, 1.0, -1.5]).double()
    got = R.loss(x, w, targets, torch.float32, weights, gradient=True)
    assert got["loss"][0][2] == 0 and got["loss"][0][4] == 0 and not bool(got["dx"][0][2].any()) and not bool(got["dx"][0][3].any())
    value = lambda x, w: float((R.loss(x, w, targets, torch.float32)["loss"][0] * weights).sum())  # noqa: E731
    for n, name in enumerate(("dx", "dw")):
        for at in ((0, 0), (1, 3), (5, 4)):
            ends = []
            for e in (1e-5, -1e-5):
                moved = [x.clone(), w.clone()]
                moved[n][at] += e
                ends.append(value(*moved))
            assert abs((ends[0] - ends[1]) / 2e-5 - float(got[name][0][at])) < 1e-6
    counts = torch.tensor([0, 1, 3, 5])
    assert torch.allclose(got["loss"][0][counts], torch.nn.functional.cross_entropy(x @ w.T, targets.where(targets < 9, 0).clamp(min=0), reduction="none")[counts])

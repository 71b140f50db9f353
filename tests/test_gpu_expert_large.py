"""Quantising and the gradient of combining at sizes that take the forms for many rows: several blocks a thread, four choices that share a token's row."""
import numpy as np
import pytest
import torch

from paper_1705_05249_amd import experts as X
from tests import expert_reference as R

pytestmark = pytest.mark.gpu
CODE = {"f32": X.MG_F32, "f16": X.MG_F16, "bf16": X.MG_BF16}
TYPE = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}


def power_of_two(e):
    """2^e as a float64, from its bits: torch's ldexp and pow are off by a last place on the GPU"""
    return ((e.long() + 1023) << 52).view(torch.float64)


def quantized(x):
    """(values of the e4m3 numbers, scales) of row blocks by the definition, in 64 bits: exact"""
    rows, cols = x.shape
    blocks = -(-cols // 128)
    v = torch.nn.functional.pad(x.double(), (0, blocks * 128 - cols)).view(rows, blocks, 128)
    part, power = torch.frexp(v.abs().amax(2))                     # largest = part * 2^power; 448 = 7/8 * 2^9
    e = torch.where(part > 0.875, power - 8, power - 9).clamp(min=-126)
    scales = torch.where(part > 0, power_of_two(e), 1.0)
    v = v / scales[:, :, None]
    _, power = torch.frexp(v.abs().clamp(min=2.0 ** -6))           # |v| is in 2^(power-1) .. 2^power, in steps of 2^(power-4)
    step = power_of_two(power - 4)
    return ((v / step).round() * step).reshape(rows, blocks * 128)[:, :cols], scales


@pytest.mark.parametrize("kind", ("f32", "f16", "bf16"))
@pytest.mark.parametrize("batch,rows,cols,pad", ((1, 16401, 1030, 0), (1, 140001, 100, 3), (3, 5511, 1025, 7), (2, 66000, 128, 0)))
def test_quantize_rows(kind, batch, rows, cols, pad):
    gen = torch.Generator(device="cuda").manual_seed(rows)
    ld, blocks = cols + pad, -(-cols // 128)
    assert batch * rows * blocks >= 131072                          # (from there on a thread takes four blocks)
    x = (torch.randn(batch, rows, ld, device="cuda", generator=gen) * torch.exp(torch.randn(rows, 1, device="cuda", generator=gen))).to(TYPE[kind])
    q = torch.full((batch, rows, ld + 1), 0xA5, dtype=torch.uint8, device="cuda")
    s = torch.full((batch, rows, blocks + 1), -3.0, device="cuda")
    X.mg_block_quantize_batched(CODE[kind], X.MG_BLOCK_ROW, batch, rows, cols, x, ld, rows * ld, q, ld + 1, rows * (ld + 1), s, blocks + 1, rows * (blocks + 1),
                                None, 0, 0, None, 0, 0)
    torch.cuda.synchronize()
    for b in range(batch):
        values, scales = quantized(x[b, :, :cols])
        assert torch.equal(q[b, :, :cols].view(torch.float8_e4m3fn).double(), values) and torch.equal(s[b, :, :blocks].double(), scales)
    assert (q[:, :, cols:] == 0xA5).all() and (s[:, :, blocks:] == -3.0).all()


def test_quantize_rows_of_experts():
    """rows fetched by the sorted index; those of no expert stay as they were"""
    rows, cols, fan, experts, total = 33000, 520, 3, 7, 32011
    gen = torch.Generator(device="cuda").manual_seed(2)
    x = torch.randn(rows // fan, cols, device="cuda", generator=gen).bfloat16()
    source = torch.full((rows,), -1, dtype=torch.int32)
    source[:total] = torch.randperm(rows)[:total].int()
    offsets = torch.tensor([0, 0, 100, 9000, 9001, 20000, 32000, total], dtype=torch.int32)
    q, s = torch.full((rows, cols), 0xA5, dtype=torch.uint8, device="cuda"), torch.full((rows, 5), -3.0, device="cuda")
    X.mg_block_quantize_grouped(X.MG_BF16, experts, offsets.cuda(), rows, cols, x, cols, source.cuda(), fan, q, cols, s, 5, None, 0, None, 0)
    torch.cuda.synchronize()
    values, scales = quantized(x[source[:total].long().cuda() // fan])
    assert torch.equal(q[:total].view(torch.float8_e4m3fn).double(), values) and torch.equal(s[:total].double(), scales)
    assert (q[total:] == 0xA5).all() and (s[total:] == -3.0).all()


@pytest.mark.parametrize("kind", ("f32", "f16", "bf16"))
@pytest.mark.parametrize("tokens,fan", ((513, 1), (600, 3), (301, 5), (270, 8), (1100, 4)))
@pytest.mark.parametrize("cols,pad", ((96, 0), (512, 5), (2051, 0), (2048, 8)))
def test_combine_gradient(kind, tokens, fan, cols, pad):
    assert tokens * -(-fan // 4) >= 512                             # (from there on four choices share the row of dO)
    unit, least = R.ROUNDOFF[kind]
    gen = torch.Generator(device="cuda").manual_seed(tokens + cols)
    rng = np.random.default_rng(tokens + cols)
    slots, ld = tokens * fan, cols + pad
    ids = rng.integers(0, 9, slots)
    ids[rng.random(slots) < 0.2] = -1
    order = np.argsort(np.where(ids < 0, 9, ids), kind="stable")
    total = int((ids >= 0).sum())
    position = np.full(slots, -1, np.int32)
    position[order[:total]] = np.arange(total)
    at = torch.tensor(position).cuda()
    g, y = (torch.randn(r, ld, device="cuda", generator=gen).to(TYPE[kind]) for r in (tokens, slots))
    y[total:] = float("nan")
    w = torch.rand(tokens, fan, device="cuda", generator=gen) - 0.5
    dy, dw = torch.full((slots, ld), 9.0, dtype=TYPE[kind], device="cuda"), torch.full((slots + 4,), 9.0, device="cuda")
    X.mg_expert_combine_grad(CODE[kind], tokens, fan, cols, g, ld, y, ld, at, w, dy, ld, dw)
    alone_y, alone_w = torch.full_like(dy, 9.0), torch.full_like(dw, 9.0)
    X.mg_expert_combine_grad(CODE[kind], tokens, fan, cols, g, ld, None, 0, at, w, alone_y, ld, None)
    X.mg_expert_combine_grad(CODE[kind], tokens, fan, cols, g, ld, y, ld, at, None, None, 0, alone_w)
    torch.cuda.synchronize()
    assert torch.equal(alone_y, dy) and torch.equal(alone_w, dw)
    assert (dy[total:] == 9.0).all() and (dy[:, cols:] == 9.0).all() and (dw[slots:] == 9.0).all()
    kept = (at >= 0).nonzero()[:, 0]
    given = g[:, :cols].double()[kept // fan]
    want = w.view(-1).double()[kept, None] * given
    got = dy[:, :cols].double()[at[kept].long()]
    assert ((got - want).abs() <= (unit + 2.0 ** -23) * want.abs() + least).all()
    terms = given * y[:, :cols].double()[at[kept].long()]
    assert ((dw[kept].double() - terms.sum(1)).abs() <= (cols + 8) * 2.0 ** -24 * terms.abs().sum(1)).all()
    assert (dw[:slots][at < 0] == 0.0).all()

"""The codes of a pool held in 4 bits on a B200, against the definition in whole fractions: steps rounded towards zero, quotients
that lie beside a half, and ranges at the ends of the types."""
import math
from fractions import Fraction

import pytest
import torch

import q4_reference as q4
from paper_2609_11744_b200 import kvc
from test_gpu_q4 import BF16, FP16

pytestmark = pytest.mark.gpu
D = 64


def down(x, dtype):
    """The largest number of the type that is at most x >= 0."""
    bits, least = (8, -133) if dtype is BF16 else (11, -24)
    if x == 0:
        return Fraction(0)
    e = 0
    while Fraction(2) ** (e + 1) <= x:
        e += 1
    while Fraction(2) ** e > x:
        e -= 1
    place = Fraction(2) ** max(e - bits + 1, least)
    return x // place * place


def group(x, dtype):
    """Codes, step and offset of 32 numbers."""
    y = [Fraction(v) for v in x]
    low = min(y)
    step = down((max(y) - low) / 15, dtype)
    return [0 if step == 0 else min(15, round((v - low) / step)) for v in y], float(step), float(low)


def written(x, dtype):
    """x [T, D] through kvc_append_q4 -> codes, step, offset of its keys and of its values."""
    t = x.shape[0]
    v = x[:, None].cuda()
    nb = -(-t // 16)
    pool = torch.zeros(1, 2, nb, 16 * q4.row_bytes(D), dtype=torch.uint8, device="cuda")
    lay = kvc.kvc_layout_create_q4(pool, 1, nb, 16, 1, D, 16)
    kvc.kvc_append_q4(lay, 0, None, v, v, None, torch.arange(t, device="cuda"), None, None)
    return [[y.reshape(nb * 16, -1)[:t].cpu() for y in q4.unpack_slabs(pool[0, p], 1, 16, D, dtype)] for p in range(2)], (lay, pool)


def check(x, dtype):
    want = [group(g.tolist(), dtype) for g in x.double().view(-1, 32)]
    codes = torch.tensor([w[0] for w in want], dtype=torch.uint8).view(-1, D)
    step, offset = (torch.tensor([w[i] for w in want], dtype=torch.float64).to(dtype).view(-1, D // 32) for i in (1, 2))
    for c, s, o in written(x, dtype)[0]:
        assert torch.equal(s, step) and torch.equal(o, offset)
        assert torch.equal(c, codes)


@pytest.mark.parametrize("dtype", [BF16, FP16])
def test_quotients_beside_a_half(dtype):
    """Offsets a hair from zero, values of k + 1/2 steps: the quotient lies beside the half by less than 32 bits can tell."""
    rows = []
    powers = (-5, -9, -14, -18, -22, -24) if dtype is FP16 else (-5, -14, -22, -24, -26, -30, -40, -80, -130)
    for p in powers:
        for sign in (1, -1):
            for unit in (1.0, 2.0**-6, 2.0**7):
                if dtype is BF16 and unit * 2.0**p < 2.0**-133:
                    continue
                low = sign * 2.0**p * (1.0 if dtype is FP16 and unit < 1 else unit)
                half = [(i + 0.5) * unit for i in range(15)]
                top = 15 * unit
                rows.append(torch.tensor([low, top] + half + [i * unit for i in range(1, 16)]))
    rows.append(torch.zeros(32))
    if len(rows) % 2:
        rows.append(torch.ones(32))
    check(torch.stack(rows).double().to(dtype).view(-1, D), dtype)


@pytest.mark.parametrize("dtype", [BF16, FP16])
def test_numbers_of_all_sizes(dtype):
    gen = torch.Generator().manual_seed(1)
    n = 240
    top, bottom = (15, -24) if dtype is FP16 else (120, -130)
    power = torch.randint(bottom, top, (n, 1), generator=gen)
    spread = torch.randint(0, 40, (n, 1), generator=gen) * torch.rand(n, 32, generator=gen)
    x = torch.randn(n, 32, generator=gen, dtype=torch.float64) * torch.exp2((power - spread).clamp(min=bottom).double())
    if dtype is FP16:
        x = x.clamp(-65504, 65504)
    # few different values a group, so that quotients of few bits, halves among them, are frequent
    x[: n // 2] = (x[: n // 2] / torch.exp2(power[: n // 2].double() - 3)).round().clamp(-64, 64) * torch.exp2(power[: n // 2].double() - 3)
    check(x.to(dtype).view(-1, D), dtype)


def test_ranges_that_no_float_has():
    """A range beyond a 32-bit float's stands for NaN; the largest that is one does not."""
    top = torch.finfo(BF16).max
    x = torch.zeros(2, D)
    x[0, 0], x[0, 5], x[0, 40], x[0, 41] = top, -top, top / 2, -top / 2
    x[1, 3], x[1, 50] = -top, top
    x = x.to(BF16)
    _, (lay, pool) = written(x, BF16)
    out = torch.zeros(2, 1, D, dtype=BF16, device="cuda")
    kvc.kvc_read_q4(lay, 0, out, None, torch.arange(2, device="cuda"))
    out = out[:, 0].float().cpu()
    assert torch.isnan(out[0, :32]).all()
    for got, g in ((out[0, 32:], x[0, 32:]), (out[1, :32], x[1, :32]), (out[1, 32:], x[1, 32:])):
        codes, step, offset = group(g.double().tolist(), BF16)
        want = torch.tensor([offset + step * c for c in codes], dtype=torch.float64).float().to(BF16).float()
        assert torch.equal(got, want) and math.isfinite(step)

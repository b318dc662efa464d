"""Attention over a pool held in 4 bits on a B200, row by row against bounds of each row's own keys: queries of
any size, and ordinary calls of few rows."""
import pytest
import torch

import q4_row_bounds as bounds
from test_gpu_q4 import BF16, FP16, Case, heads

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [BF16, FP16])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("lens,new,h,block,window,sinks", [
    ([1, 2, 127, 129, 700], [1] * 5, 2, 16, 0, 0), ([3000, 40], [2, 1], 3, 8, 100, 5), ([500, 9], [4, 3], 1, 16, 0, 0), ([900], [1], 7, 24, 64, 70)])
def test_ordinary_calls(dtype, d, lens, new, h, block, window, sinks):
    hq, hkv = heads(h)
    c = Case(dtype, lens, new, hq, hkv, d, block, seed=len(lens) + block, extra=300 // block + 1)
    want = bounds.attention(c, window, sinks)
    bounds.check(c, c.run(window, sinks, hint=max(new)), want, "few")


@pytest.mark.parametrize("dtype,q_power", [(FP16, -6), (FP16, -10), (FP16, -16), (FP16, 8), (BF16, -30), (BF16, -90), (BF16, 30), (BF16, 70)])
@pytest.mark.parametrize("d,lens,new,h", [(128, [512, 3], [1, 1], 2), (64, [512, 70], [2, 1], 0), (128, [300, 129, 264], [100, 60, 3], 4), (64, [600], [500], 2), (128, [900], [30], 1)])
def test_queries_of_any_size(dtype, q_power, d, lens, new, h):
    """Scores of the same size from queries of any: what a row's log-sum-exp is off by does not change."""
    hq, hkv = heads(h)
    c = Case(dtype, lens, new, hq, hkv, d, 16, seed=2, extra=9)
    c.q = (c.q.float() * 2.0**q_power).to(dtype)
    scale = d ** -0.5 * 2.0**-q_power
    want = bounds.attention(c, scale=min(scale, 1e18))
    got = c.run(hint=max(new), scale=min(scale, 1e18))
    bounds.check(c, got, want, "few" if max(new) * hq // hkv <= 16 else "many")


@pytest.mark.parametrize("dtype", [BF16, FP16])
@pytest.mark.parametrize("new,h", [(1, 0), (2, 0), (40, 2), (300, 4)])
def test_rows_of_queries_of_different_sizes(dtype, new, h):
    hq, hkv = heads(h)
    c = Case(dtype, [400, new + 65], [new, new], hq, hkv, 128, 16, seed=4, extra=9)
    top = 8 if dtype is FP16 else 40
    power = torch.arange(c.t * hq).view(c.t, hq) * 7 % (2 * top + 1) - top
    c.q = torch.ldexp(c.q.float(), power.cuda()[..., None]).to(dtype)
    c.q[0, 0] = 0
    c.q[0, -1, 1:] = 0
    for scale in (128**-0.5 * 2.0**-top, 128**-0.5 * 2.0**(16 - top)):   # (scores up to 2^20: 32 bits tell no more apart than that)
        want = bounds.attention(c, scale=scale)
        bounds.check(c, c.run(hint=new, scale=scale), want, "few" if new * hq // hkv <= 16 else "many")

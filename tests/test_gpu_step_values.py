"""Values at the edges of a step's types: infinities, NaN and negative zeros in queries and keys."""
import math

import pytest
import torch

import step_reference as ref
from paper_2609_11744_b200 import kvc
from test_gpu_step import BF16, FP16, make_layout

pytestmark = pytest.mark.gpu


def same(got, want):
    """Equal, NaN with NaN, zeros with their signs."""
    return bool((got.isnan() == want.isnan()).all()) and torch.equal(got.nan_to_num(7.0, 8.0, 9.0), want.nan_to_num(7.0, 8.0, 9.0)) and \
        torch.equal(got.signbit() & ~got.isnan(), want.signbit() & ~want.isnan())


@pytest.mark.parametrize("dtype", [BF16, FP16])
@pytest.mark.parametrize("d,rot", [(128, 0), (64, 0), (128, 64), (80, 16), (256, 96)])
@pytest.mark.parametrize("interleaved", [False, True])
def test_append_keeps_values_outside_the_rotation_to_themselves(dtype, d, rot, interleaved):
    """Without a norm what is not rotated is copied, whatever stands beside it; what is rotated is its pair's alone."""
    t, hq, hkv, block = 70, 6, 2, 16
    g = torch.Generator().manual_seed(d + rot)
    q, k, v = (torch.randn(t, h, d, generator=g) for h in (hq, hkv, hkv))
    for x in (q, k):
        odd = torch.tensor([math.inf, -math.inf, math.nan, -0.0, 0.0])
        at = torch.rand(x.shape, generator=g)
        x[at < 0.15] = odd[torch.randint(0, 5, x.shape, generator=g)][at < 0.15]
    q, k, v = (x.to(dtype).cuda() for x in (q, k, v))
    pool = torch.zeros(1, 2, 8, block, hkv, d, dtype=dtype, device="cuda")
    out = torch.zeros_like(q)
    positions = torch.randint(1, 50, (t,), generator=g, dtype=torch.int32).cuda()
    angle = torch.arange(50.0)[:, None] * 0.7 ** torch.arange(max(rot // 2, 1))
    table = torch.cat([angle.cos(), angle.sin()], 1).cuda()
    kvc.kvc_append(make_layout(pool, block), 0, q, k, v, out, torch.arange(t).cuda(), positions if rot else None, table if rot else None,
                   interleaved=interleaved)
    for got, x in ((out, q), (pool.view(2, -1, hkv, d)[0, :t], k)):
        assert same(got[..., rot:], x[..., rot:])
        if rot:
            want = ref.norm_rotate(x, None, 0.0, positions, table, rot, interleaved)[..., :rot]
            a = got[..., :rot].double()
            special = ~want.isfinite()
            assert same(a[special], want[special])
            # two products, a sum and the rounding to the type
            size = ref.norm_rotate(x, None, 0.0, positions, None, 0, False).abs().nan_to_num(0.0, 0.0, 0.0).amax(-1, keepdim=True)
            bound = torch.finfo(dtype).eps / 2 * want.abs() + 2.0**-22 * size + 2.0**-25
            assert ((a - want).abs() <= bound)[~special].all()


@pytest.mark.parametrize("dtype", [BF16, FP16])
def test_append_norm_of_a_head_with_an_infinity(dtype):
    """The mean of squares is infinite: every finite value of that head becomes zero, the infinity NaN, other heads are as
    they are without it."""
    t, hkv, d, block = 9, 3, 128, 16
    g = torch.Generator().manual_seed(4)
    k = torch.randn(t, hkv, d, generator=g).to(dtype).cuda()
    w = torch.rand(d, generator=g).add(0.5).to(dtype).cuda()
    got = []
    for bad in (False, True):
        pool = torch.zeros(1, 2, 4, block, hkv, d, dtype=dtype, device="cuda")
        x = k.clone()
        if bad:
            x[4, 1, 17] = math.inf
        kvc.kvc_append(make_layout(pool, block), 0, None, x, k, None, torch.arange(t).cuda(), None, None, k_weight=w)
        got.append(pool.view(2, -1, hkv, d)[0, :t].clone())
    assert got[1][4, 1, 17].isnan() and (got[1][4, 1, :17] == 0).all() and (got[1][4, 1, 18:] == 0).all()
    rest = torch.ones(t, hkv, dtype=torch.bool)
    rest[4, 1] = False
    assert torch.equal(got[0][rest.cuda()], got[1][rest.cuda()])


def test_append_of_two_rows_to_one_slot_leaves_elements_of_either():
    """And what other slots get is not touched by it."""
    t, hkv, d, block = 64, 2, 128, 16
    pool = torch.zeros(1, 2, 8, block, hkv, d, dtype=BF16, device="cuda")
    x = torch.arange(1, t + 1, device="cuda")[:, None, None].expand(t, hkv, d).to(BF16).contiguous()
    slots = torch.arange(t).cuda()
    slots[32:] = slots[:32].flip(0)   # rows i and 63 - i
    kvc.kvc_append(make_layout(pool, block), 0, None, x, -x, None, slots, None, None)
    for got, sign in zip(pool.view(2, -1, hkv, d), (1.0, -1.0)):
        first, second = x[:32] * sign, x[32:].flip(0) * sign
        assert ((got[:32] == first) | (got[:32] == second)).all() and (got[32:] == 0).all()

"""Plain forms of a pool held in 4 bits and of attention over it, for tests: 64-bit arithmetic that shares nothing
with the library."""
import math

import torch

GROUP = 32


def row_bytes(d):
    return d // 2 + d // 8


def quantise(x):
    """x [..., D] of a 16-bit type -> (codes uint8 [..., D], step, offset [..., D / 32] of the type)."""
    dt = x.dtype
    y = x.double().unflatten(-1, (-1, GROUP))
    low, high = y.amin(-1), y.amax(-1)
    step = ((high - low).float() / 15).double()            # a 32-bit quotient, as the definition's range is
    bits, least = (8, -133) if dt is torch.bfloat16 else (11, -24)
    place = torch.ldexp(torch.ones_like(step), (torch.frexp(step).exponent - bits).clamp(min=least))
    step = torch.floor(step / place) * place               # towards zero
    safe = torch.where(step > 0, step, torch.ones_like(step))[..., None]
    code = ((y - low[..., None]) / safe).round().clamp(0, 15)
    code = torch.where(step[..., None] > 0, code, torch.zeros_like(code))
    return code.flatten(-2).to(torch.uint8), step.to(dt), low.to(dt)


def pack_slabs(codes, step, offset):
    """codes [..., block, head, D], step and offset [..., block, head, D / 32] -> bytes [..., slab]."""
    c = codes.transpose(-2, -3)
    data = (c[..., 0::2] | c[..., 1::2] << 4).contiguous()
    scales = torch.stack([step.transpose(-2, -3), offset.transpose(-2, -3)], -1).contiguous().view(torch.uint8)
    return torch.cat([data.flatten(-2), scales.flatten(-3)], -1).flatten(-2)


def unpack_slabs(slabs, heads, block, d, dtype):
    """bytes [..., slab] -> (codes, step, offset) as pack_slabs takes them."""
    rows = slabs.unflatten(-1, (heads, block * row_bytes(d)))
    data = rows[..., : block * d // 2].unflatten(-1, (block, d // 2))
    codes = torch.stack([data & 15, data >> 4], -1).flatten(-2).transpose(-2, -3)
    scales = rows[..., block * d // 2:].contiguous().view(dtype).unflatten(-1, (block, d // GROUP, 2)).transpose(-3, -4)
    return codes, scales[..., 0], scales[..., 1]


def values(codes, step, offset):
    """What codes stand for, in 64 bits."""
    return (offset.double()[..., None] + step.double()[..., None] * codes.double().unflatten(-1, (-1, GROUP))).flatten(-2)


def pool_of(x):
    """x [..., block, head, D] -> bytes [..., slab]."""
    return pack_slabs(*quantise(x))


def attention(q, parts, tables, rows, lens, block, scale, window=0, sinks=0):
    """q [T, Hq, D]; parts: for K and V (codes, step, offset) of the blocks, [NB, block, Hkv, ..]; rows[r]: (first, last + 1).

    Returns (out, lse, weight, slips): weight is sum_j softmax_j |v_j|; slips bound the error of a score, in the two kinds of
    kernel that may serve a call:
      few rows   2^-23 * 40 * scale * sum_d |q_d| (143 * step + |offset|): 36 sums of 32 products with codes that carry a bias of
                 128 at most (codes end at 15) and 4 of the groups, each cut to 2^-23 of the largest
      many       scale * sum_d |q_d k_d| (eps / 2 + 2^-23 (D + 8)): k rounded to the type, D products
    with, as a third, keys times the largest |v|, for weights below fp16's normal range."""
    t, hq, d = q.shape
    dt = q.dtype
    dev = q.device
    half = torch.finfo(dt).eps / 2
    out = torch.zeros(t, hq, d, dtype=torch.float64, device=dev)
    lse = torch.full((t, hq), -math.inf, dtype=torch.float64, device=dev)
    weight = torch.zeros_like(out)
    slip_few, slip_many, small = 0.0, 0.0, 0.0
    qd = q.double()
    for r, (a, b) in enumerate(rows):
        n = int(lens[r])
        if b <= a or n <= 0:
            continue
        ids = tables[r].to(dev).long()
        j = torch.arange(min(n, ids.numel() * block), device=dev)
        at, ok = ids[j // block], None
        ok = (at >= 0) & (at < parts[0][0].shape[0])
        at = torch.where(ok, at, torch.zeros_like(at))
        (kc, ks, ko), (vc, vs, vo) = [[x[at, j % block] for x in p] for p in parts]
        k, v = values(kc, ks, ko), values(vc, vs, vo)                   # [key, Hkv, D]
        hkv = k.shape[1]
        g = hq // hkv
        p = torch.arange(n - (b - a), n, device=dev)[:, None]
        see = (j <= p) & ok
        if window:
            see &= (p - j < window) | (j < sinks)
        size = (143 * ks.double().abs() + ko.double().abs()).repeat_interleave(GROUP, -1)
        for h in range(hkv):
            x = qd[a:b, h * g: (h + 1) * g]
            s = (torch.einsum("tgd,kd->gtk", x, k[:, h]) * scale).masked_fill(~see, -math.inf)
            some = see.any(-1)
            z = torch.logsumexp(s, -1)
            w = torch.exp(s - torch.where(some, z, torch.zeros_like(z))[..., None]).masked_fill(~see, 0.0)
            vv = torch.where(ok[:, None], v[:, h], torch.zeros_like(v[:, h]))
            out[a:b, h * g: (h + 1) * g] = (w @ vv).transpose(0, 1)
            weight[a:b, h * g: (h + 1) * g] = (w @ vv.abs()).transpose(0, 1)
            lse[a:b, h * g: (h + 1) * g] = z.transpose(0, 1)
            if len(j):
                few = torch.einsum("tgd,kd->gtk", x.abs(), size[:, h]).masked_fill(~see, 0.0).amax() * 40 * 2.0**-23
                many = torch.einsum("tgd,kd->gtk", x.abs(), k[:, h].abs()).masked_fill(~see, 0.0).amax() * (half + (d + 8) * 2.0**-23)
                slip_few, slip_many = max(slip_few, float(few) * scale), max(slip_many, float(many) * scale)
                small = max(small, len(j) * float(vv.abs().max()))
    return out, lse, weight, (slip_few, slip_many, small)


def bounds(dtype, out, lse, weight, slips, few=False):
    """(bound of out, bound of lse); few: the kernel for few rows is known to serve.  The result's rounding: half of eps of it.  Each weight's and each value's rounding to the
    type: half of eps each of sum w|v|.  A score's slip: a factor exp(+-slip) on a weight and on their sum, twice slip to
    first order (and half its square again).  32-bit sums and exponentials: 2^-16 together.  In fp16 a weight below the
    normal range is off by up to 2^-25 instead, and the sum of weights is at least 1: 2^-25 max|v| a key."""
    slip, small = slips[0] if few else max(slips[:2]), slips[2]
    half = torch.finfo(dtype).eps / 2
    extra = 2.0**-25 * small if dtype is torch.float16 else 0.0
    b_out = half * out.abs() + weight * (2 * half + 2 * slip + slip * slip + 2.0**-16) * 1.01 + extra + 2.0**-24
    b_lse = slip + 2.0**-18 + lse.abs().nan_to_num(posinf=0.0) * 2.0**-21
    return b_out, b_lse

"""Plain 64-bit forms of the operators of a serving step, for tests: loops over requests, rows and
heads that share nothing with the library."""
import math

import numpy as np
import torch


def map_tokens(ctx, new, free, tables, block, max_blocks, num_blocks, capacity):
    """(tables, cu, positions, slots, request, total, counts) as numpy arrays."""
    tables = tables.copy()
    cu, taken, refused = [0], 0, 0
    pos, slot, req = [], [], []
    for r in range(len(ctx)):
        c = max(0, int(ctx[r]))
        n = max(0, min(int(new[r]), 2**31 - 1 - c))
        have = min(-(-c // block), max_blocks)
        need = min(-(-(c + n) // block), max_blocks) if n else have
        for b in range(have, need):
            if taken < len(free):
                tables[r, b] = free[taken]
            else:
                tables[r, b] = -1
            taken += 1
        for i in range(n):
            p = c + i
            b = p // block
            pos.append(p)
            req.append(r)
            covered = b < max_blocks and (b < -(-c // block) or tables[r, b] != -1)
            if not covered:
                refused += 1
            ok = b < max_blocks and 0 <= tables[r, b] < num_blocks
            slot.append(int(tables[r, b]) * block + p % block if ok else -1)
        cu.append(cu[-1] + n)
    total = [max(0, int(c)) + max(0, min(int(n), 2**31 - 1 - max(0, int(c)))) for c, n in zip(ctx, new)]

    def fit(v, fill):
        return np.array((v + [fill] * capacity)[:capacity], dtype=np.int64)

    return (tables, np.array(cu), fit(pos, 0), fit(slot, -1), fit(req, -1), np.array(total, dtype=np.int64),
            np.array([cu[-1], min(taken, len(free)), refused]))


def norm_rotate(x, weight, eps, positions, cos_sin, rot, interleaved):
    """x [T, H, D] -> float64 [T, H, D]."""
    y = x.double()
    if weight is not None:
        y = y / torch.sqrt((y * y).mean(-1, keepdim=True) + eps) * weight.double()
    if not rot:
        return y
    row = cos_sin.double()[positions.long()][:, None]
    z = y.clone()
    for n in range(rot // 2):
        i, j = (2 * n, 2 * n + 1) if interleaved else (n, n + rot // 2)
        c, s = row[..., n], row[..., rot // 2 + n]
        z[..., i] = y[..., i] * c - y[..., j] * s
        z[..., j] = y[..., j] * c + y[..., i] * s
    return z


def attention(q, keys, values, rows, lens, scale, window=0, sinks=0):
    """q [T, Hq, D]; keys[r], values[r] [len_r, Hkv, D] per request; rows: (first, last+1) of each request.

    Returns (out, lse, weight, slip): `weight` is sum_j softmax_j |v_j|, the size that a relative error
    of the weights is multiplied by; `slip` bounds the error of a 32-bit score,
    (D + 4) * 2^-24 * scale * max_j sum |q k|: D products added one after the other, two roundings of
    the scaling, and two of the subtraction of the maximum."""
    t, hq, d = q.shape
    out = torch.zeros(t, hq, d, dtype=torch.float64)
    lse = torch.full((t, hq), -math.inf, dtype=torch.float64)
    weight = torch.zeros(t, hq, d, dtype=torch.float64)
    slip = 0.0
    q = q.double().cpu()
    for r, (a, b) in enumerate(rows):
        k, v = keys[r].double().cpu(), values[r].double().cpu()
        n = k.shape[0]
        g = hq // k.shape[1]
        for i in range(a, b):
            p = int(lens[r]) - (b - a) + (i - a)
            j = torch.arange(n)
            see = j <= p
            if window:
                see &= (p - j < window) | (j < sinks)
            see = see.nonzero()[:, 0]
            if not len(see):
                continue
            for h in range(hq):
                kk, vv = k[see, h // g], v[see, h // g]
                s = (kk @ q[i, h]) * scale
                slip = max(slip, float((kk.abs() @ q[i, h].abs()).max()) * scale * (d + 4) * 2.0**-24)
                lse[i, h] = torch.logsumexp(s, 0)
                w = torch.exp(s - lse[i, h])
                out[i, h] = w @ vv
                weight[i, h] = w @ vv.abs()
    return out, lse, weight, slip


def attention_bounds(dtype, out, lse, weight, slip):
    """(bound of out, bound of lse).  Errors of the result: its own rounding, eps/2 of it; the rounding of
    each weight to the pool's type, eps/2 of it, so eps/2 of sum w|v|; the scores' slip, a factor
    exp(+-slip) on each weight and on their sum, twice slip to first order; and 32-bit sums and exponentials
    (2^-22 each, and up to a few hundred additions at 2^-24): 2^-16 together.  A weight below fp16's normal
    range is off by at most 2^-25 instead, and the largest weight of a row is 1, so the sum of weights is at
    least 1: 2^-25 times the largest |v| times the number of keys, for which 2^-12 max|v| stands up to 8192 keys."""
    half = torch.finfo(dtype).eps / 2
    extra = 2.0**-12 * float(weight.max()) if dtype is torch.float16 else 0.0
    b_out = half * out.abs() + weight * (half + 2 * slip + 2.0**-16) * 1.01 + extra * half * 16 + 2.0**-25
    b_lse = slip + 2.0**-18 + lse.abs().nan_to_num(posinf=0.0) * 2.0**-21
    return b_out, b_lse

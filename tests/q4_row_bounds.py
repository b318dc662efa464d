"""Bounds of attention over a pool held in 4 bits, row by row, for tests: 64-bit arithmetic that shares nothing with the
library.

What a row's error may come from, with w the softmax, half = eps / 2 of the type, and all sums in 32 bits:
  result      half of |out|
  weights     half of each, values half of each: 2 * half * sum w |v|; in fp16 a weight below the normal range is off by 2^-25
              instead, and their sum is at least 1
  exponentials and sums of them  2^-16 of sum w |v|, 2^-18 + |lse| 2^-21 of the log-sum-exp
  scores      a slip of e moves a weight by a factor exp(+-e), and their sum; the log-sum-exp by e.  e is the largest of the
              row's own keys:
    few rows    codes are exact, queries too: scale * sum_d |q_d| (15 step + |offset|) times 40 * 2^-23, for 36 sums of 32 products
                and 4 of the groups, each cut to 2^-23 of the largest
    many rows   keys are rounded to 11 bits: scale * sum_d |q_d| (2^-12 |k_d| + a) and D + 8 cuts of 2^-23 of sum_d |q_d k_d|.
                a: fp16's smallest numbers, 2^-25 of a key's rounding in fp16; in bf16 a step (times 15), an offset and the sum each,
                17 * 2^-25
    and rows that see few keys  twice as many products, of the key and of what its rounding left: 2^-22 |k_d| + 2^-25"""
import math

import torch

from q4_reference import GROUP, values

FEW_KEYS = 64


def attention(c, window=0, sinks=0, scale=None):
    """c: a Case.  -> out, lse, weight [T, Hq, D], and the slips of few rows, of many, and of many with few keys in sight
    [T, Hq], keys in sight [T], keys times the largest |v| [T, Hq]."""
    q, d, block, hkv = c.q.double(), c.d, c.block, c.hkv
    t, hq, dev = q.shape[0], q.shape[1], q.device
    g, scale = hq // hkv, scale or d ** -0.5
    bf16 = c.dtype is torch.bfloat16
    out = torch.zeros(t, hq, d, dtype=torch.float64, device=dev)
    weight = torch.zeros_like(out)
    lse = torch.full((t, hq), -math.inf, dtype=torch.float64, device=dev)
    few, many, exact, small = (torch.zeros(t, hq, dtype=torch.float64, device=dev) for _ in range(4))
    seen = torch.zeros(t, dtype=torch.long, device=dev)
    for r, n in enumerate(c.lens):
        a, b = c.cu[r], c.cu[r + 1]
        ids = c.tables[r, : c.wide].to(dev).long()
        j = torch.arange(min(max(n, 0), len(ids) * block), device=dev)
        if b <= a or len(j) == 0:
            continue
        (kc, ks, ko), (vc, vs, vo) = [[x[ids[j // block], j % block] for x in p] for p in c.parts]
        k, v = values(kc, ks, ko), values(vc, vs, vo)                   # [key, Hkv, D]
        size = (15 * ks.double() + ko.double().abs()).repeat_interleave(GROUP, -1)
        p = torch.arange(n - (b - a), n, device=dev)[:, None]
        see = j <= p
        if window:
            see &= (p - j < window) | (j < sinks)
        seen[a:b] = see.sum(-1)
        for h in range(hkv):
            x = q[a:b, h * g: (h + 1) * g]
            s = (torch.einsum("tgd,kd->tgk", x, k[:, h]) * scale).masked_fill(~see[:, None], -math.inf)
            some = see.any(-1)[:, None]
            z = torch.logsumexp(s, -1)
            w = torch.exp(s - torch.where(some, z, 0.0)[..., None]).masked_fill(~see[:, None], 0.0)
            at = (slice(a, b), slice(h * g, (h + 1) * g))
            out[at], weight[at], lse[at] = w @ v[:, h], w @ v[:, h].abs(), z
            small[at] = see.sum(-1)[:, None] * v[:, h].abs().max()
            most = lambda e: (e * scale).masked_fill(~see[:, None], 0.0).amax(-1)
            both, one = torch.einsum("tgd,kd->tgk", x.abs(), k[:, h].abs()), x.abs().sum(-1, keepdim=True)
            few[at] = most(torch.einsum("tgd,kd->tgk", x.abs(), size[:, h]) * (40 * 2.0**-23))
            many[at] = most(both * (2.0**-12 + (d + 8) * 2.0**-23) + one * (17 if bf16 else 1) * 2.0**-25)
            exact[at] = most(both * (2.0**-22 + (2 * d + 16) * 2.0**-23) + one * 2.0**-25)
    return out, lse, weight, few, many, exact, seen, small


def check(c, got, want, kind):
    """kind: "few" or "many", the kernel that serves the call, or "any"."""
    out, lse = got
    w_out, w_lse, weight, few, many, exact, seen, small = want
    many = torch.where((seen <= FEW_KEYS)[:, None], exact, many)
    slip = few if kind == "few" else many if kind == "many" else torch.maximum(few, many)
    half = torch.finfo(c.dtype).eps / 2
    e = slip[..., None]
    b_out = half * w_out.abs() + weight * (2 * half + 2 * e + e * e + 2.0**-16) * 1.01 + 2.0**-24
    if c.dtype is torch.float16:
        b_out = b_out + 2.0**-25 * small[..., None]
    none = torch.isinf(w_lse)
    b_lse = slip + 2.0**-18 + w_lse.abs().masked_fill(none, 0.0) * 2.0**-21
    assert torch.isfinite(out).all() and (out[none] == 0).all() and torch.equal(torch.isinf(lse), none)
    worst = ((lse.double() - w_lse).abs() / b_lse)[~none].max()
    assert worst <= 1, ("lse", float(worst))
    worst = ((out.double() - w_out).abs() / b_out).max()
    assert worst <= 1, ("out", float(worst))

"""More operators of a serving step over the paged pool, for measurement: their cases, plain forms and exact values.

A cache held in 4 bits, the attention that reads it, and rotary positions with several axes:

  axes      norms, rotation by positions with several axes, and the write of K and V into a pool of 16-bit elements
  store4    the same write into a pool held in 4 bits, and the tokens read back as the values that the pool stands for
  attend4   causal attention over a pool held in 4 bits, with an optional sliding window and first tokens that stay visible
  shared4   the same for requests that share a long prefix, whose keys and values are read once per group

A row of the 4-bit pool is one token of one KV head: D codes of 4 bits in groups of 32 values, and for each group a step
and an offset in the model's 16-bit type; a value is offset + step * code.  In a block the rows of a KV head lie
together: [kv head][token][D / 2 bytes of codes], behind each head's codes its [token][D / 32][step, offset].

With ``own`` false, ``run`` computes an operator from elementary torch operations in 32 bits; with ``own`` true it
calls the library.
"""
import math
import random

import numpy as np
import torch

own = False

DT = {"bf16": torch.bfloat16, "fp16": torch.float16}
GROUP = 32


# ------------------------------------------------------------------ cases
def listed():
    return [
        # decode tokens of the 8B shape behind images: time, height and width in sections of a head's pairs
        dict(name="axes_decode_64", op="axes", tokens=64, hq=32, hkv=8, d=128, rot=128, pairs="halves", norm=True,
             axes="sections", n_axes=3, dtype="bf16", block=16, far=8192, seed=1),
        # the patches of one picture, an odd number, small heads: two axes that take turns over neighbouring pairs
        dict(name="axes_patches_5041", op="axes", tokens=5041, hq=12, hkv=4, d=64, rot=64, pairs="neighbours", norm=False,
             axes="turns", n_axes=2, dtype="fp16", block=16, far=256, seed=2),
        # a prefill step of the 70B-class shape with pictures in it
        dict(name="axes_prefill_16384", op="axes", tokens=16384, hq=64, hkv=8, d=128, rot=128, pairs="halves", norm=True,
             axes="sections", n_axes=3, dtype="bf16", block=16, far=32768, seed=3),
        # decode tokens of the 8B shape into a 4-bit pool
        dict(name="store4_decode_64", op="store4", tokens=64, hq=32, hkv=8, d=128, rot=128, pairs="halves", norm=True,
             axes="one", n_axes=1, dtype="bf16", block=16, far=80000, seed=4),
        # an odd number of tokens, small heads, part of the head rotated
        dict(name="store4_odd_1003", op="store4", tokens=1003, hq=12, hkv=4, d=64, rot=32, pairs="neighbours", norm=True,
             axes="one", n_axes=1, dtype="fp16", block=16, far=8192, seed=5),
        # a prefill step of the 70B-class shape into a 4-bit pool
        dict(name="store4_prefill_16384", op="store4", tokens=16384, hq=64, hkv=8, d=128, rot=128, pairs="halves", norm=True,
             axes="one", n_axes=1, dtype="bf16", block=16, far=32768, seed=6),
        # the smallest attention call: one token of one request with an 8192-token context, 8B shape
        dict(name="attend4_one_8192", op="attend4", requests=1, q="one", ctx="fixed", length=8192, hq=32, hkv=8, d=128,
             window=0, sinks=0, dtype="bf16", block=16, seed=7),
        # one decode step of the benchmark's batch: 64 requests, lognormal contexts, 70B-class heads
        dict(name="attend4_decode_64", op="attend4", requests=64, q="one", ctx="lognormal", length=32768, hq=64, hkv=8,
             d=128, window=0, sinks=0, dtype="bf16", block=16, seed=8),
        # ragged prompts behind cached contexts, small heads, an odd window
        dict(name="attend4_ragged_window", op="attend4", requests=9, q="ragged", ctx="lognormal", length=4096, hq=12, hkv=4,
             d=64, window=1000, sinks=5, dtype="fp16", block=16, seed=9),
        # the whole 8192-token prompt of the 8B shape
        dict(name="attend4_prefill_8192", op="attend4", requests=1, q="all", ctx="fixed", length=8192, hq=32, hkv=8, d=128,
             window=0, sinks=0, dtype="bf16", block=16, seed=10),
        # 64 requests that share the benchmark's 1024-token prefix
        dict(name="shared4_64x1024", op="shared4", requests=64, groups=1, prefix=1024, length=1024, hq=64, hkv=8, d=128,
             dtype="bf16", block=16, seed=11),
        # 32 questions about one 32k-token document
        dict(name="shared4_32x32k", op="shared4", requests=32, groups=1, prefix=32000, length=333, hq=32, hkv=8, d=128,
             dtype="fp16", block=16, seed=12),
    ]


def _spread(rng, low, high):
    """A whole number between the two, spread over its logarithm."""
    return int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))


def draw(rng):
    op = rng.choice(["axes", "store4", "attend4", "attend4", "shared4"])
    hq, hkv, d = rng.choice([(32, 8, 128), (64, 8, 128), (12, 4, 64), (8, 1, 128), (7, 1, 64), (16, 16, 64), (28, 4, 128),
                             (5, 5, 128), (40, 2, 64)])
    dtype = rng.choice(["bf16", "fp16"])
    block = rng.choice([8, 16, 16, 16, 24, 32, 64])
    seed = rng.randrange(1 << 20)
    if op in ("axes", "store4"):
        axes = rng.choice(["sections", "turns"] if op == "axes" else ["one", "one", "sections"])
        return dict(op=op, tokens=_spread(rng, 1, 8192), hq=hq, hkv=hkv, d=d, rot=rng.choice([d, d, d // 2, 16]),
                    pairs=rng.choice(["halves", "neighbours"]), norm=rng.random() < 0.75, axes=axes,
                    n_axes=1 if axes == "one" else rng.choice([2, 3, 3, 4]), dtype=dtype, block=block,
                    far=_spread(rng, 16, 80000), seed=seed)
    if op == "attend4":
        window = rng.choice([0, 0, _spread(rng, 1, 4096)])
        sinks = rng.choice([0, 1, 4, 64, 100]) if window else 0
        kind = rng.choice(["one", "few", "ragged"])
        if kind == "ragged":
            return dict(op=op, requests=_spread(rng, 1, 12), q="ragged", ctx="lognormal", length=_spread(rng, 64, 4096),
                        hq=hq, hkv=hkv, d=d, window=window, sinks=sinks, dtype=dtype, block=block, seed=seed)
        return dict(op=op, requests=_spread(rng, 1, 64), q=kind, ctx=rng.choice(["fixed", "lognormal"]),
                    length=_spread(rng, 1, 16000), hq=hq, hkv=hkv, d=d, window=window, sinks=sinks, dtype=dtype,
                    block=block, seed=seed)
    requests = _spread(rng, 2, 48)
    return dict(op=op, requests=requests, groups=rng.randint(1, max(1, requests // 4)), prefix=_spread(rng, 16, 16000),
                length=_spread(rng, 1, 1000), hq=hq, hkv=hkv, d=d, dtype=dtype, block=block, seed=seed)


# ------------------------------------------------------------------ sizes of a case (host side, as a scheduler has them)
def _lengths(case):
    """(context tokens, new tokens) of every request, as a scheduler knows them."""
    rng = np.random.default_rng(case["seed"])
    n = case["requests"]
    if case["op"] == "shared4":
        rest = rng.integers(max(1, case["length"] // 2), case["length"] + 1, n)
        return case["prefix"] + rest - 1, np.ones(n, np.int64)
    total = np.full(n, case["length"], np.int64)
    if case["ctx"] == "lognormal":
        median = max(1, case["length"] // 16) if case["length"] > 8192 else max(1, case["length"] // 2)
        total = np.clip(np.exp(rng.normal(math.log(median), 1.0, n)), min(case["length"], 128), case["length"]).astype(np.int64)
    if case["q"] == "one":
        new = np.ones(n, np.int64)
    elif case["q"] == "few":             # a few drafted tokens at once
        new = np.minimum(rng.integers(1, 6, n), total)
    elif case["q"] == "all":
        new = total.copy()
    else:
        new = np.maximum(1, (total * rng.random(n)).astype(np.int64))
    return total - new, new


def _groups(case):
    """Where each group of requests begins, and behind the last one."""
    rng = np.random.default_rng(case["seed"] + 1)
    cuts = np.sort(rng.choice(np.arange(1, case["requests"]), case["groups"] - 1, replace=False)) if case["groups"] > 1 else []
    return np.concatenate([[0], cuts, [case["requests"]]]).astype(np.int64)


def _pairs(case):
    """(query, key) pairs that are visible, and keys that some query of their request sees."""
    ctx, new = _lengths(case)
    window, sinks = case.get("window", 0), case.get("sinks", 0)
    pairs = keys = 0
    for c, n in zip(ctx.tolist(), new.tolist()):
        p = np.arange(c, c + n, dtype=np.int64)
        if window:
            pairs += int((np.minimum(p + 1, window) + np.clip(p + 1 - window, 0, sinks)).sum())
            first = max(0, c + 1 - window)
            keys += c + n - first + min(first, sinks)
        else:
            pairs += int((p + 1).sum())
            keys += c + n
    return pairs, keys


def _pair_axes(case):
    """The axis of every pair of a head."""
    n, a = case["rot"] // 2, case["n_axes"]
    if case["axes"] == "turns":
        return [i % a for i in range(n)]
    # sections: the first axis (time) has the smallest share, as where three axes split 64 pairs into 16, 24 and 24
    first = n // (a + 1) if a > 1 else n
    return [0 if i < first else 1 + (i - first) * (a - 1) // (n - first) for i in range(n)]


def work(case):
    d, hq, hkv = case["d"], case["hq"], case["hkv"]
    row = d // 2 + d // 8
    if case["op"] in ("axes", "store4"):
        t = case["tokens"]
        moved = 2 * t * (hq + 2 * hkv) * d + 4 * t * case["rot"] + (8 + 4 * case["n_axes"]) * t
        moved += 2 * t * hq * d + 2 * t * hkv * 2 * d          # queries; keys and values (read back, of a 4-bit pool)
        if case["op"] == "store4":
            moved += 2 * t * hkv * row
        return {"bytes": moved, "flops": t * (hq + hkv) * d * 8}
    pairs, keys = _pairs(case)
    t = int(_lengths(case)[1].sum())
    if case["op"] == "shared4":
        keys -= case["prefix"] // case["block"] * case["block"] * (case["requests"] - case["groups"])
    return {"bytes": 2 * keys * hkv * row + 4 * t * hq * d + 4 * t * hq + 4 * (keys // case["block"]),
            "flops": 4 * pairs * hq * d}


# ------------------------------------------------------------------ the 4-bit form, from elementary operations
def _quantise(x):
    """x [..., D] of a 16-bit type -> (codes [..., D] uint8, step [..., D / 32], offset [..., D / 32] of that type)."""
    y = x.float().unflatten(-1, (-1, GROUP))
    low, high = y.amin(-1), y.amax(-1)
    exact_step = (high - low) / 15
    step = exact_step.to(x.dtype)                               # rounded towards zero
    bits = step.view(torch.int16)
    step = torch.where(step.float() > exact_step, bits - 1, bits).view(x.dtype)
    s = step.float()[..., None]
    code = torch.where(s > 0, ((y - low[..., None]) / torch.where(s > 0, s, 1.0)).round(), torch.zeros_like(y)).clamp(max=15)
    return code.flatten(-2).to(torch.uint8), step, low.to(x.dtype)


def _stand_for(codes, step, offset):
    """The values of the codes, in 32 bits."""
    c = codes.unflatten(-1, (-1, GROUP)).float()
    return (offset.float()[..., None] + step.float()[..., None] * c).flatten(-2)


def _pack_pool(x):
    """x [..., block, token, kv head, D] -> the pool's bytes [..., block, slab]."""
    codes, step, offset = _quantise(x.transpose(-2, -3))        # [..., block, head, token, D]
    data = (codes[..., 0::2] | codes[..., 1::2] << 4).flatten(-2)
    scales = torch.stack([step, offset], -1).contiguous().view(torch.uint8).flatten(-3)
    return torch.cat([data, scales], -1).flatten(-2)


def _unpack_blocks(blocks, hkv, tokens, d, dtype, wide=torch.float32):
    """Bytes [..., slab] of blocks -> values [..., head, token, D]."""
    rows = blocks.unflatten(-1, (hkv, -1))
    data = rows[..., : tokens * d // 2].unflatten(-1, (tokens, -1))
    scales = rows[..., tokens * d // 2:].contiguous().view(dtype).unflatten(-1, (tokens, -1, 2))
    codes = torch.stack([data & 15, data >> 4], -1).flatten(-2).unflatten(-1, (-1, GROUP)).to(wide)
    return codes.mul_(scales[..., :1].to(wide)).add_(scales[..., 1:].to(wide)).flatten(-2)


# ------------------------------------------------------------------ inputs
def _ints(a, dtype=torch.int32):
    return torch.as_tensor(np.ascontiguousarray(a), dtype=dtype, device="cuda")


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)

    def normal(*shape, dtype):
        return torch.randn(*shape, generator=gen, device="cuda", dtype=dtype)

    block, dtype, d, hq, hkv = case["block"], DT[case["dtype"]], case["d"], case["hq"], case["hkv"]
    if case["op"] in ("axes", "store4"):
        t, rot, far, axes = case["tokens"], case["rot"], case["far"], case["n_axes"]
        blocks = -(-t // block) + 3
        qkv = normal(t, (hq + 2 * hkv) * d, dtype=dtype)
        positions = torch.randint(0, far, (axes, t), generator=gen, device="cuda", dtype=torch.int32)
        slots = torch.randperm(blocks * block, generator=gen, device="cuda")[:t]
        angle = torch.arange(far, device="cuda", dtype=torch.float64)[:, None] * (
            500000.0 ** (-torch.arange(0, rot, 2, device="cuda", dtype=torch.float64) / rot))
        s = dict(op=case["op"], q=qkv[:, : hq * d].view(t, hq, d), k=qkv[:, hq * d: (hq + hkv) * d].view(t, hkv, d),
                 v=qkv[:, (hq + hkv) * d:].view(t, hkv, d), q_out=torch.zeros(t, hq, d, dtype=dtype, device="cuda"),
                 positions=positions, slots=slots, table=torch.cat([angle.cos(), angle.sin()], 1).float(),
                 q_weight=1 + 0.1 * normal(d, dtype=dtype) if case["norm"] else None,
                 k_weight=1 + 0.1 * normal(d, dtype=dtype) if case["norm"] else None, eps=1e-6,
                 rot=rot, neighbours=case["pairs"] == "neighbours", axes=_ints(_pair_axes(case), torch.int64))
        if case["op"] == "axes":
            s["pool"] = normal(2, 2, blocks, block, hkv, d, dtype=dtype)
        else:
            s["k_out"], s["v_out"] = (torch.zeros(t, hkv, d, dtype=dtype, device="cuda") for _ in range(2))
        if own:
            from paper_2609_11744_b200 import kvc
            s["pair_axis"] = bytes(_pair_axes(case)) if axes > 1 else None
            if case["op"] == "axes":
                s["layout"] = kvc.kvc_layout_create_dense(s["pool"], 2, 2, blocks, block, hkv, d, 2, block)
            else:
                s["pool"] = torch.zeros(2, 2, blocks, block * hkv * d * 5 // 8, dtype=torch.uint8, device="cuda")
                s["layout"] = kvc.kvc_layout_create_q4(s["pool"], 2, blocks, block, hkv, d, block)
        return s
    ctx, new = _lengths(case)
    total = ctx + new
    n, t, need = len(ctx), int(new.sum()), -(-total // block)
    wide = int(need.max())
    group_at = _groups(case) if case["op"] == "shared4" else None
    blocks = int(need.sum()) + 5
    pool = torch.zeros(2, 2, blocks, block * hkv * d * 5 // 8, dtype=torch.uint8, device="cuda")
    step = max(1, (1 << 26) // (block * hkv * d))
    for plane in range(2):                                      # the second layer's, which the calls read
        for at in range(0, blocks, step):
            pool[1, plane, at: at + step] = _pack_pool(normal(min(step, blocks - at), block, hkv, d, dtype=dtype))
    ids = torch.randperm(blocks, generator=gen, device="cuda").int()
    tables = torch.zeros(n, wide, dtype=torch.int32, device="cuda")
    rows = np.concatenate([r * wide + np.arange(k) for r, k in enumerate(need)])
    tables.view(-1)[_ints(rows, torch.int64)] = ids[: len(rows)]
    s = dict(op=case["op"], pool=pool, tables=tables, lens=_ints(total), cu=_ints(np.concatenate([[0], np.cumsum(new)])),
             q=normal(t, hq, d, dtype=dtype), out=torch.zeros(t, hq, d, dtype=dtype, device="cuda"),
             lse=torch.zeros(t, hq, dtype=torch.float32, device="cuda"), scale=d ** -0.5, window=case.get("window", 0),
             sinks=case.get("sinks", 0), longest_q=int(new.max()), longest=int(total.max()), block=block, hkv=hkv)
    if group_at is not None:
        first = group_at[np.searchsorted(group_at, np.arange(n), side="right") - 1]   # the first request of each group
        shared = case["prefix"] // block                                              # whole blocks are shared
        tables[:, :shared] = tables[_ints(first, torch.int64), :shared]
        s["group_starts"] = _ints(group_at)
        s["prefix_lens"] = _ints(np.full(case["groups"], shared * block))
    if own:
        from paper_2609_11744_b200 import kvc
        s["layout"] = kvc.kvc_layout_create_q4(pool, 2, blocks, block, hkv, d, block)
        size = kvc.kvc_attention_q4_workspace_bytes(s["layout"], t, n, hq, 0 if group_at is None else case["groups"])
        s["workspace"] = torch.empty(size, dtype=torch.uint8, device="cuda")
    return s


# ------------------------------------------------------------------ plain forms
def _turn(x, weight, s):
    """Norm over each head in 32 bits, then the rotation of its first `rot` values, each pair by its own axis' position."""
    x = x.float()
    if weight is not None:
        x = x * torch.rsqrt(x.square().mean(-1, keepdim=True) + s["eps"]) * weight.float()
    rot = s["rot"]
    at = s["positions"].long()[s["axes"]].t()                   # [token, pair]
    cos = s["table"][:, : rot // 2].gather(0, at)[:, None]
    sin = s["table"][:, rot // 2:].gather(0, at)[:, None]
    if s["neighbours"]:
        a, b = x[..., 0:rot:2], x[..., 1:rot:2]
        turned = torch.stack([a * cos - b * sin, b * cos + a * sin], -1).flatten(-2)
    else:
        a, b = x[..., : rot // 2], x[..., rot // 2: rot]
        turned = torch.cat([a * cos - b * sin, b * cos + a * sin], -1)
    return torch.cat([turned, x[..., rot:]], -1)


def _axes_plain(s):
    pool = s["pool"]
    keys, values = pool[1, 0].view(-1, *pool.shape[-2:]), pool[1, 1].view(-1, *pool.shape[-2:])
    s["q_out"].copy_(_turn(s["q"], s["q_weight"], s))
    keys[s["slots"]] = _turn(s["k"], s["k_weight"], s).to(pool.dtype)
    values[s["slots"]] = s["v"]
    return [s["q_out"], pool[1, 0], pool[1, 1]]


def _store_plain(s):
    s["q_out"].copy_(_turn(s["q"], s["q_weight"], s))
    s["k_out"].copy_(_stand_for(*_quantise(_turn(s["k"], s["k_weight"], s).to(s["k"].dtype))))
    s["v_out"].copy_(_stand_for(*_quantise(s["v"].contiguous())))
    return [s["q_out"], s["k_out"], s["v_out"]]


def _attend_plain(s):
    """All requests at once, padded to the longest: scores, masked softmax and the weighted sum, in 32 bits."""
    q, pool, tables, lens, cu, block, hkv = s["q"], s["pool"], s["tables"].long(), s["lens"], s["cu"], s["block"], s["hkv"]
    n, most, longest = tables.shape[0], s["longest_q"], s["longest"]
    hq, d = q.shape[1], q.shape[2]

    def plane(p):                                               # [request, head, key, D]
        x = _unpack_blocks(pool[1, p][tables], hkv, block, d, q.dtype)
        return x.transpose(1, 2).reshape(n, hkv, -1, d)[:, :, :longest]

    i = torch.arange(most, device="cuda", dtype=torch.int32)
    j = torch.arange(longest, device="cuda", dtype=torch.int32)
    count = cu[1:] - cu[:-1]
    row = torch.where(i < count[:, None], cu[:-1, None] + i, q.shape[0]).long()      # a row of no token behind the last
    g = hq // hkv
    x = torch.cat([q, q[:1]])[row].view(n, most, hkv, g, d).permute(0, 2, 1, 3, 4).reshape(n, hkv, most * g, d).float()
    p = (lens - count)[:, None] + i
    seen = j <= p[..., None]
    if s["window"]:
        seen &= (p[..., None] - j < s["window"]) | (j < s["sinks"])
    seen = seen[:, None, :, None].expand(n, 1, most, g, longest).reshape(n, 1, most * g, longest)
    score = (x @ plane(0).transpose(-1, -2)) * s["scale"]
    score.masked_fill_(~seen, -math.inf)
    top = score.amax(-1, keepdim=True)
    score = score.sub_(top).exp_()
    total = score.sum(-1, keepdim=True)
    o = (score @ plane(1) / total).view(n, hkv, most, g, d).permute(0, 2, 1, 3, 4).reshape(n, most, hq, d)
    lse = (top + total.log()).view(n, hkv, most, g).permute(0, 2, 1, 3).reshape(n, most, hq)
    out = torch.cat([s["out"], s["out"][:1]])
    out[row] = o.to(q.dtype)
    s["out"].copy_(out[:-1])
    tall = torch.cat([s["lse"], s["lse"][:1]])
    tall[row] = lse
    s["lse"].copy_(tall[:-1])
    return [s["out"], s["lse"]]


def run(state):
    s = state
    if own:
        from paper_2609_11744_b200 import kvc
        if s["op"] == "axes":
            kvc.kvc_append_axes(s["layout"], 1, s["q"], s["k"], s["v"], s["q_out"], s["slots"], s["positions"], s["table"],
                                s["pair_axis"], q_weight=s["q_weight"], k_weight=s["k_weight"], eps=s["eps"],
                                interleaved=s["neighbours"])
            return [s["q_out"], s["pool"][1, 0], s["pool"][1, 1]]
        if s["op"] == "store4":
            kvc.kvc_append_q4(s["layout"], 1, s["q"], s["k"], s["v"], s["q_out"], s["slots"], s["positions"], s["table"],
                              pair_axis=s["pair_axis"], q_weight=s["q_weight"], k_weight=s["k_weight"], eps=s["eps"],
                              interleaved=s["neighbours"])
            kvc.kvc_read_q4(s["layout"], 1, s["k_out"], s["v_out"], s["slots"])
            return [s["q_out"], s["k_out"], s["v_out"]]
        if s["op"] == "attend4":
            kvc.kvc_attention_q4(s["layout"], 1, s["q"], s["out"], s["tables"], s["lens"], s["cu"], s["workspace"],
                                 scale=s["scale"], window=s["window"], sinks=s["sinks"], lse=s["lse"],
                                 max_q_len=s["longest_q"])
            return [s["out"], s["lse"]]
        kvc.kvc_attention_q4_shared(s["layout"], 1, s["q"], s["out"], s["tables"], s["lens"], s["cu"], s["group_starts"],
                                    s["prefix_lens"], s["workspace"], scale=s["scale"], lse=s["lse"],
                                    max_q_len=s["longest_q"])
        return [s["out"], s["lse"]]
    if s["op"] == "axes":
        return _axes_plain(s)
    if s["op"] == "store4":
        return _store_plain(s)
    return _attend_plain(s)


# ------------------------------------------------------------------ exact values
def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] in ("axes", "store4"):
        rot, half = s["rot"], s["rot"] // 2
        first = torch.arange(0, rot, 2, device="cuda") if s["neighbours"] else torch.arange(half, device="cuda")
        second = first + 1 if s["neighbours"] else first + half

        def value(x, weight):
            y = x.double()
            if weight is not None:
                y = y / torch.sqrt((y * y).sum(-1, keepdim=True) / y.shape[-1] + s["eps"]) * weight.double()
            z = y.clone()
            # the table is an input: its 32-bit values are taken as they are
            for n, axis in enumerate(s["axes"].tolist()):
                row = s["positions"][axis].long()
                c, w = s["table"][row, n].double()[:, None], s["table"][row, half + n].double()[:, None]
                i, j = int(first[n]), int(second[n])
                z[..., i] = y[..., i] * c - y[..., j] * w
                z[..., j] = y[..., j] * c + y[..., i] * w
            return z

        if case["op"] == "axes":
            planes = s["pool"][1].double()
            flat = planes.view(2, -1, *planes.shape[-2:])
            flat[0, s["slots"]] = value(s["k"], s["k_weight"])
            flat[1, s["slots"]] = s["v"].double()
            return [value(s["q"], s["q_weight"]), planes[0], planes[1]]

        def held(x):
            """What the codes of x, rounded to the model's type, stand for."""
            dt = s["k"].dtype
            y = x.to(dt).double().view(*x.shape[:-1], -1, GROUP)
            low = y.min(-1, keepdim=True).values
            step = (y.max(-1, keepdim=True).values - low) / 15
            # rounded towards zero to the type's bits: 8 of bf16, 11 of fp16, or its last place for the smallest
            bits, least = (8, -133) if dt is torch.bfloat16 else (11, -24)
            place = torch.ldexp(torch.ones_like(step), (torch.frexp(step).exponent - bits).clamp(min=least))
            down = torch.floor(step / place) * place
            code = torch.where(down > 0, (y - low) / torch.where(down > 0, down, torch.ones_like(down)), torch.zeros_like(y))
            return (low + down * torch.round(code).clamp(0, 15)).view(x.shape)

        return [value(s["q"], s["q_weight"]), held(value(s["k"], s["k_weight"])), held(s["v"].double())]
    block, hkv, d = case["block"], case["hkv"], case["d"]
    g = case["hq"] // hkv
    ctx, new = _lengths(case)
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    lse = torch.zeros(s["lse"].shape, dtype=torch.float64, device="cuda")

    def values(blocks):
        """[key, head, D] of a request's blocks."""
        rows = blocks.view(len(blocks), hkv, block * (d // 2 + d // 8))
        data = rows[..., : block * d // 2].reshape(len(blocks), hkv, block, d // 2)
        scale = rows[..., block * d // 2:].reshape(len(blocks), hkv, block, -1).view(s["q"].dtype).double()
        x = torch.empty(len(blocks), hkv, block, d, dtype=torch.float64, device="cuda")
        x[..., 0::2] = (data % 16).double()
        x[..., 1::2] = (data // 16).double()
        x = x * scale[..., 0::2].repeat_interleave(GROUP, -1) + scale[..., 1::2].repeat_interleave(GROUP, -1)
        return x.transpose(1, 2).reshape(-1, hkv, d)

    at = 0
    for r in range(len(ctx)):
        c, m = int(ctx[r]), int(new[r])
        used = s["tables"][r, : -(-(c + m) // block)].long()
        k, v = (values(s["pool"][1, p][used])[: c + m] for p in range(2))
        for lo in range(0, m, 1024):
            hi = min(m, lo + 1024)
            p = torch.arange(c + lo, c + hi, device="cuda")[:, None]
            j = torch.arange(c + m, device="cuda")[None]
            hidden = j > p
            if s["window"]:
                hidden = hidden | ((j <= p - s["window"]) & (j >= s["sinks"]))
            for h in range(hkv):
                x = s["q"][at + lo: at + hi, h * g: (h + 1) * g].double()
                y = torch.einsum("tgd,kd->gtk", x, k[:, h]) * s["scale"]
                y = y.masked_fill(hidden[None], -math.inf)
                z = torch.logsumexp(y, -1)
                o = torch.exp(y - z[..., None]) @ v[:, h]
                out[at + lo: at + hi, h * g: (h + 1) * g] = o.transpose(0, 1)
                lse[at + lo: at + hi, h * g: (h + 1) * g] = z.transpose(0, 1)
        at += m
    return [out, lse]

"""Positions with several axes and pools held in 4 bits on a B200, against 64-bit arithmetic: rotation by axes, the
write in 4 bits, the way back, attention over it alone and with shared prefixes, and a step of them together with
pack and unpack."""
import math

import pytest
import torch

import q4_reference as q4
import step_reference as ref
from paper_2609_11744_b200 import kvc

pytestmark = pytest.mark.gpu
BF16, FP16 = torch.bfloat16, torch.float16
I32 = dict(dtype=torch.int32, device="cuda")


def bits(x):
    return x.contiguous().view(torch.uint8)


def angles(rows, rot, base=10000.0):
    a = torch.arange(float(rows), dtype=torch.float64)[:, None] * base ** (-torch.arange(0, max(rot, 1), 2, dtype=torch.float64) / max(rot, 1))
    return torch.cat([a.cos(), a.sin()], 1).float().cuda()


def heads_of(t, hq, hkv, d, dtype, gen, gap=8):
    """q, k, v as parts of one packed row, with a gap behind it."""
    qkv = torch.randn(t, (hq + 2 * hkv) * d + gap, generator=gen).to(dtype).cuda()
    return [qkv[:, a * d: b * d].view(t, b - a, d) if b > a else None for a, b in ((0, hq), (hq, hq + hkv), (hq + hkv, hq + 2 * hkv))]


# ------------------------------------------------------------------ positions with several axes
def split(kind, n_axes, pairs, gen):
    if kind == "turns":
        return bytes(i % n_axes for i in range(pairs))
    if kind == "any":
        return bytes(torch.randint(0, n_axes, (pairs,), generator=gen).tolist())
    return bytes(i * n_axes // pairs for i in range(pairs))


@pytest.mark.parametrize("dtype", [BF16, FP16])
@pytest.mark.parametrize("t,hq,hkv,d,rot,interleaved,norm,n_axes,kind", [
    (1, 32, 8, 128, 128, False, True, 3, "sections"), (67, 12, 4, 64, 64, True, True, 2, "turns"), (33, 7, 1, 80, 80, False, True, 4, "any"),
    (130, 5, 5, 96, 16, False, False, 3, "turns"), (41, 16, 2, 256, 256, False, True, 3, "sections"), (9, 3, 1, 200, 96, True, True, 4, "any"),
    (19, 0, 2, 128, 64, False, True, 3, "turns"), (2100, 8, 1, 128, 128, False, True, 3, "sections"), (5, 2, 1, 16, 16, True, True, 1, "sections")])
def test_append_axes(dtype, t, hq, hkv, d, rot, interleaved, norm, n_axes, kind):
    gen = torch.Generator().manual_seed(t + d)
    block, rows = 16, 300
    nb = -(-t // block) + 2
    pool = torch.randn(2, 2, nb, block, hkv, d, generator=gen).to(dtype).cuda()
    before = pool.clone()
    lay = kvc.kvc_layout_create_dense(pool, 2, 2, nb, block, hkv, d, 2, block)
    q, k, v = heads_of(t, hq, hkv, d, dtype, gen)
    out = torch.full((t, hq, d), 7.0, dtype=dtype, device="cuda") if hq else None
    slots = torch.randperm(nb * block, generator=gen)[:t]
    positions = torch.randint(0, rows, (n_axes, t), generator=gen, dtype=torch.int32)
    skip, lost = torch.zeros(t, dtype=torch.bool), 0
    if t > 8:
        slots[2] = -1
        slots[5] = nb * block
        positions[n_axes - 1, 7] = rows          # behind the table on one axis
        positions[0, 8] = -1
        skip[[2, 5, 7, 8]], lost = True, 3
    table = angles(rows, rot)
    w = [(1 + 0.2 * torch.randn(d, generator=gen)).to(dtype).cuda() if norm else None for _ in range(2)]
    axis = split(kind, n_axes, rot // 2, gen)
    kvc.kvc_append_axes(lay, 1, q, k, v, out, slots.cuda(), positions.cuda(), table, axis, q_weight=w[0], k_weight=w[1], eps=1e-5,
                        interleaved=interleaved)
    torch.cuda.synchronize()
    assert kvc.kvc_poll_device_status(lay) == (lost, 0)
    half, keep = torch.finfo(dtype).eps / 2, ~skip
    at = positions.long().clamp(0, rows - 1).cuda()

    def want(x, weight):
        y = x.double()
        if weight is not None:
            y = y / torch.sqrt((y * y).mean(-1, keepdim=True) + 1e-5) * weight.double()
        z, size = y.clone(), y.abs()
        for n in range(rot // 2):
            i, j = (2 * n, 2 * n + 1) if interleaved else (n, n + rot // 2)
            c, s = table.double()[at[axis[n]], n][:, None], table.double()[at[axis[n]], rot // 2 + n][:, None]
            z[..., i] = y[..., i] * c - y[..., j] * s
            z[..., j] = y[..., j] * c + y[..., i] * s
            size[..., i] = size[..., j] = y[..., i].abs() + y[..., j].abs()
        return z, size

    kk = keep.cuda()

    def near(got, x, weight):
        # its own rounding, and 32-bit arithmetic: a sum of d squares, its root, six products and sums, on the size of both terms
        z, size = want(x, weight)
        return ((got.double() - z[kk]).abs() <= half * z[kk].abs() * 1.01 + size[kk] * (d + 16) * 2.0**-24 + 2.0**-24).all()

    if hq:
        assert near(out[kk], q, w[0]) and (out[~kk] == 7).all()
    flat = pool.view(2, 2, nb * block, hkv, d)
    good = slots[keep].cuda()
    assert near(flat[1, 0, good], k, w[1])
    assert torch.equal(flat[1, 1, good], v[kk])
    rest = torch.ones(nb * block, dtype=torch.bool)
    rest[slots[keep]] = False
    assert torch.equal(bits(flat[1][:, rest]), bits(before.view(2, 2, -1, hkv, d)[1][:, rest])) and torch.equal(bits(flat[0]), bits(before.view(2, 2, -1, hkv, d)[0]))


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("d,rot", [(128, 128), (64, 32)])
def test_axes_of_one_position_are_kvc_append(interleaved, d, rot):
    gen = torch.Generator().manual_seed(5)
    t, hq, hkv, nb = 77, 6, 3, 9
    q, k, v = heads_of(t, hq, hkv, d, BF16, gen)
    pos = torch.randint(0, 99, (t,), generator=gen, dtype=torch.int32).cuda()
    slots = torch.randperm(nb * 16, generator=gen)[:t].cuda()
    table = angles(99, rot)
    # (a table whose rows are not 16 bytes apart from a 16-byte boundary goes another way)
    loose = torch.zeros(99 * rot + 1, device="cuda")[1:].view(99, rot).copy_(table)
    results = []
    for tab, axes in ((table, None), (table, kvc.kvc_pair_axes([rot // 2 - 5, 3, 2])), (table, split("turns", 4, rot // 2, gen)), (loose, split("any", 3, rot // 2, gen))):
        pool = torch.zeros(1, 2, nb, 16, hkv, d, dtype=BF16, device="cuda")
        lay = kvc.kvc_layout_create_dense(pool, 1, 2, nb, 16, hkv, d, 2, 16)
        out = torch.zeros(t, hq, d, dtype=BF16, device="cuda")
        if axes is None:
            kvc.kvc_append(lay, 0, q, k, v, out, slots, pos, tab, interleaved=interleaved)
        else:
            kvc.kvc_append_axes(lay, 0, q, k, v, out, slots, pos.expand(max(axes) + 1, t).contiguous(), tab, axes, interleaved=interleaved)
        results.append((out, pool))
    for out, pool in results[1:]:
        assert torch.equal(out, results[0][0]) and torch.equal(pool, results[0][1])


# ------------------------------------------------------------------ the write in 4 bits, and the way back
def q4_layout(pool, block, hkv, d, order="dense"):
    layers, planes, nb, slab = pool.shape
    if order == "planes":
        return kvc.kvc_layout_create(layers, 2, nb, block, hkv, q4.row_bytes(d), 1, block, plane_ptrs=[pool[i, j] for i in range(layers) for j in range(2)])
    return kvc.kvc_layout_create_q4(pool, layers, nb, block, hkv, d, block)


@pytest.mark.parametrize("dtype", [BF16, FP16])
@pytest.mark.parametrize("t,hq,hkv,d,rot,interleaved,norm,block,axes", [
    (1, 32, 8, 128, 128, False, True, 16, 1), (1, 1, 2, 64, 0, False, False, 2, 1), (3, 4, 4, 64, 64, True, True, 16, 1), (67, 12, 4, 64, 32, True, True, 24, 2),
    (33, 7, 1, 128, 128, False, True, 1, 1), (130, 5, 5, 128, 16, False, False, 8, 1), (19, 0, 2, 128, 64, False, True, 3, 3), (700, 28, 4, 128, 128, True, False, 64, 1),
    (41, 16, 2, 64, 16, False, True, 16, 3), (45, 3, 3, 64, 48, False, True, 32, 1), (61, 2, 7, 128, 96, False, True, 16, 1), (2100, 8, 1, 128, 0, False, True, 16, 1)])
def test_append_q4_holds_what_kvc_append_would(dtype, t, hq, hkv, d, rot, interleaved, norm, block, axes):
    gen = torch.Generator().manual_seed(t + d + rot)
    nb, rows = -(-t // block) + 4, 500
    q, k, v = heads_of(t, hq, hkv, d, dtype, gen)
    slots = torch.randperm(nb * block, generator=gen)[:t]
    positions = torch.randint(0, rows, (axes, t), generator=gen, dtype=torch.int32)
    skip, lost = torch.zeros(t, dtype=torch.bool), 0
    if t > 8:
        slots[3], slots[5] = -1, nb * block
        skip[[3, 5]], lost = True, 1
        if rot:
            positions[axes - 1, 7] = rows
            skip[7], lost = True, 2
    table = angles(rows, rot) if rot else None
    w = [(1 + 0.2 * torch.randn(d, generator=gen)).to(dtype).cuda() if norm else None for _ in range(2)]
    kw = dict(q_weight=w[0], k_weight=w[1], eps=1e-5, interleaved=interleaved)
    axis = split("any", axes, rot // 2, gen)
    pos = positions.cuda() if rot else None
    # what a pool of 16-bit elements holds
    wide = torch.zeros(2, 2, nb, block, hkv, d, dtype=dtype, device="cuda")
    q_wide, out = (torch.full((t, hq, d), 7.0, dtype=dtype, device="cuda") if hq else None for _ in range(2))
    kvc.kvc_append_axes(kvc.kvc_layout_create_dense(wide, 2, 2, nb, block, hkv, d, 2, block), 1, q, k, v, q_wide, slots.cuda(), pos, table, axis, **kw)
    pool = torch.randint(0, 256, (2, 2, nb, block * hkv * q4.row_bytes(d)), generator=gen, dtype=torch.uint8).cuda()
    before = pool.clone()
    lay = q4_layout(pool, block, hkv, d, "planes" if t % 2 else "dense")
    kvc.kvc_append_q4(lay, 1, q, k, v, out, slots.cuda(), pos if axes > 1 or pos is None else pos[0], table, pair_axis=axis if axes > 1 else None, **kw)
    torch.cuda.synchronize()
    assert kvc.kvc_poll_device_status(lay) == (lost, 0)
    if hq:
        assert torch.equal(out, q_wide)
    good = slots[~skip].cuda()
    for p in range(2):
        want = q4.quantise(wide.view(2, 2, nb * block, hkv, d)[1, p, good])
        got = [x.reshape(nb * block, hkv, -1)[good] for x in q4.unpack_slabs(pool[1, p], hkv, block, d, dtype)]
        for a, b in zip(got, want):
            assert torch.equal(a, b)
        # the error that the header promises
        x = wide.view(2, 2, nb * block, hkv, d)[1, p, good].double()
        room = x.unflatten(-1, (-1, 32))
        room = (room.amax(-1) - room.amin(-1)).repeat_interleave(32, -1) / 30 + 15 * 2.0**-24
        assert ((q4.values(*got) - x).abs() <= room).all()
    # everything else is as it was
    restored = pool.clone()
    for p in range(2):
        # (steps and offsets of random bytes may be NaN: compared as what they are made of)
        now, old = ([x.reshape(nb * block, hkv, -1).contiguous() for x in q4.unpack_slabs(y[1, p], hkv, block, d, torch.int16)] for y in (pool, before))
        for x, y in zip(now, old):
            x[good] = y[good]
        restored[1, p] = q4.pack_slabs(*[x.view(nb, block, hkv, -1) for x in now])
    assert torch.equal(restored, before)


@pytest.mark.parametrize("dtype", [BF16, FP16])
@pytest.mark.parametrize("d", [64, 128])
def test_values_at_the_ends_of_the_type(dtype, d):
    top, tiny = torch.finfo(dtype).max, 2.0**-24 if dtype is FP16 else 2.0**-133
    rows = [torch.zeros(d), torch.full((d,), -3.25), torch.linspace(-1, 1, d), torch.arange(d) % 16 * 1.0, (torch.arange(d) % 2) * 1.0,
            torch.arange(d) * tiny, (torch.arange(d) % 16) * 3 * tiny, -torch.arange(d).double() * 2.0**-14, torch.linspace(60000, 65504, d)]
    if dtype is FP16:
        rows.append(torch.linspace(-top, top, d))
    else:
        rows.append(torch.linspace(-1e38, 1e38, d))
    # ties: differences of k + 1/2 steps, steps being exact
    rows.append(torch.tensor([0.0, 15.0] + [i + 0.5 for i in range(15)] + [3.0] * 15).repeat(d // 32))
    x = torch.stack([r.double() for r in rows]).to(dtype).cuda()
    t = len(rows)
    v = x[:, None].contiguous()
    pool = torch.zeros(1, 2, 2, 16 * q4.row_bytes(d), dtype=torch.uint8, device="cuda")
    lay = q4_layout(pool, 16, 1, d)
    slots = torch.arange(t, device="cuda") + 3
    kvc.kvc_append_q4(lay, 0, None, v, v, None, slots, None, None)
    k_out, v_out = (torch.full((t, 1, d), 5.0, dtype=dtype, device="cuda") for _ in range(2))
    kvc.kvc_read_q4(lay, 0, k_out, v_out, slots)
    want = q4.quantise(v)
    for p in range(2):
        got = [y.reshape(32, 1, -1)[slots] for y in q4.unpack_slabs(pool[0, p], 1, 16, d, dtype)]
        for a, b in zip(got, want):
            assert torch.equal(a, b)
    back = q4.values(*want).float().to(dtype)
    assert torch.equal(k_out, back) and torch.equal(v_out, back) and torch.isfinite(back).all()


@pytest.mark.parametrize("dtype", [BF16, FP16])
def test_groups_that_are_not_finite(dtype):
    d, inf, nan = 128, math.inf, math.nan
    x = torch.randn(6, 1, d, generator=torch.Generator().manual_seed(1)).to(dtype)
    for r, (at, what) in enumerate([(3, inf), (40, -inf), (70, nan), (127, inf), (0, nan)]):
        x[r, 0, at] = what
    x[4, 0, 31] = -inf
    x = x.cuda()
    pool = torch.zeros(1, 2, 1, 16 * q4.row_bytes(d), dtype=torch.uint8, device="cuda")
    lay = q4_layout(pool, 16, 1, d)
    slots = torch.arange(6, device="cuda")
    kvc.kvc_append_q4(lay, 0, None, x, x, None, slots, None, None)
    k_out, v_out = torch.zeros_like(x), torch.zeros_like(x)
    kvc.kvc_read_q4(lay, 0, k_out, v_out, slots)
    bad = ~torch.isfinite(x).unflatten(-1, (-1, 32)).all(-1).repeat_interleave(32, -1)
    clean = torch.where(bad, torch.zeros_like(x), x)
    want = q4.values(*q4.quantise(clean)).float().to(dtype)
    for out in (k_out, v_out):
        assert torch.isnan(out[bad]).all() and torch.equal(out[~bad], want[~bad])


@pytest.mark.parametrize("dtype", [BF16, FP16])
@pytest.mark.parametrize("t,hkv,d,block,which", [(1, 1, 64, 2, "kv"), (5, 8, 128, 16, "k"), (333, 3, 64, 24, "v"), (50, 40, 128, 3, "kv"), (1000, 5, 128, 16, "kv")])
def test_read_q4(dtype, t, hkv, d, block, which):
    gen = torch.Generator().manual_seed(t)
    nb = -(-t // block) + 2
    x = torch.randn(2, nb, block, hkv, d, generator=gen).to(dtype).cuda()
    pool = torch.zeros(2, 2, nb, block * hkv * q4.row_bytes(d), dtype=torch.uint8, device="cuda")
    pool[1] = q4.pool_of(x)
    lay = q4_layout(pool, block, hkv, d)
    slots = torch.randint(0, nb * block, (t,), generator=gen)     # the same slot may come twice
    keep, lost = torch.ones(t, dtype=torch.bool), 0
    if t > 4:
        slots[1], slots[4], keep[[1, 4]], lost = -5, nb * block + 9, False, 1
    wide = torch.full((2, t, hkv, d + 8), 3.0, dtype=dtype, device="cuda")
    outs = [wide[p, :, :, :d] if "kv"[p] in which else None for p in range(2)]
    kvc.kvc_read_q4(lay, 1, *outs, slots.cuda())
    torch.cuda.synchronize()
    assert kvc.kvc_poll_device_status(lay) == (lost, 0)
    want = q4.values(*q4.quantise(x)).float().to(dtype).view(2, nb * block, hkv, d)
    for p in range(2):
        if outs[p] is not None:
            assert torch.equal(outs[p][keep.cuda()], want[p][slots[keep].cuda()]) and (outs[p][~keep.cuda()] == 3).all()
        else:
            assert (wide[p] == 3).all()
    assert (wide[..., d:] == 3).all()


# ------------------------------------------------------------------ attention
class Case:
    """A pool, tables and queries; `lens` in the cache, `new` query rows of each request."""

    def __init__(self, dtype, lens, new, hq, hkv, d, block, seed=0, extra=0, shared=()):
        self.gen = g = torch.Generator().manual_seed(seed)
        self.dtype, self.lens, self.new, self.block, self.hkv, self.d, self.hq = dtype, lens, new, block, hkv, d, hq
        need = [-(-max(n, 0) // block) for n in lens]
        self.nb = nb = sum(need) + 3
        wide = max(need + [1]) + extra
        ids = torch.randperm(nb, generator=g).tolist()
        self.tables = torch.full((len(lens), wide + 2), -9, dtype=torch.int32)
        for r, n in enumerate(need):
            for b in range(n):
                self.tables[r, b] = ids.pop()
        for first, last, blocks in shared:
            self.tables[first:last, :blocks] = self.tables[first, :blocks]
        self.wide = wide
        x = torch.randn(2, nb, block, hkv, d, generator=g)
        x[0] *= 1.5
        x[1] += 0.25 * torch.randn(hkv, d, generator=g)          # offsets that are not those of the groups alone
        self.parts = [[y.cuda() for y in q4.quantise(x[p].to(dtype))] for p in range(2)]
        self.pool = torch.zeros(2, 2, nb, block * hkv * q4.row_bytes(d), dtype=torch.uint8, device="cuda")
        for p in range(2):
            self.pool[1, p] = q4.pack_slabs(*self.parts[p])
        self.cu = [0]
        for n in new:
            self.cu.append(self.cu[-1] + n)
        t = self.cu[-1]
        self.q = torch.randn(t, hq, d, generator=g).to(dtype).cuda()
        self.lay = q4_layout(self.pool, block, hkv, d)
        self.t = t

    def run(self, window=0, sinks=0, hint=0, groups=None, tail=0, lse=True, scale=None):
        out = torch.full((self.t + tail, self.hq, self.d), 9.0, dtype=self.dtype, device="cuda")
        stat = torch.full((self.t + tail, self.hq), 9.0, device="cuda") if lse else None
        q = torch.cat([self.q, torch.full((tail, self.hq, self.d), math.nan, dtype=self.dtype, device="cuda")])
        ws = torch.full((kvc.kvc_attention_q4_workspace_bytes(self.lay, self.t + tail, len(self.lens), self.hq, len(groups[1]) if groups else 0),), 255,
                        dtype=torch.uint8, device="cuda")
        tables = self.tables.cuda()[:, : self.wide]
        args = (self.lay, 1, q, out, tables, torch.tensor(self.lens, **I32), torch.tensor(self.cu, **I32))
        if groups:
            kvc.kvc_attention_q4_shared(*args, torch.tensor(groups[0], **I32), torch.tensor(groups[1], **I32), ws, lse=stat, max_q_len=hint, scale=scale)
        else:
            kvc.kvc_attention_q4(*args, ws, window=window, sinks=sinks, lse=stat, max_q_len=hint, scale=scale)
        torch.cuda.synchronize()
        if tail:
            assert (out[self.t:] == 9).all() and (stat is None or (stat[self.t:] == 9).all())
        return out[: self.t], None if stat is None else stat[: self.t]

    def want(self, window=0, sinks=0, scale=None):
        rows = list(zip(self.cu, self.cu[1:]))
        return q4.attention(self.q, self.parts, self.tables[:, : self.wide], rows, self.lens, self.block, scale or self.d ** -0.5, window, sinks)

    def check(self, got, want, few=False):
        out, lse = got
        w_out, w_lse, weight, slips = want
        b_out, b_lse = q4.bounds(self.dtype, w_out, w_lse, weight, slips, few)
        assert not torch.isnan(out).any()
        worst = ((out.double() - w_out).abs() / b_out).max()
        assert worst <= 1, worst
        none = torch.isinf(w_lse)
        assert (out[none] == 0).all()
        if lse is not None:
            assert torch.equal(torch.isinf(lse), none) and (lse[none] < 0).all()
            assert ((lse.double() - w_lse).abs()[~none] <= b_lse[~none]).all()


def heads(i):
    return [(8, 1), (4, 4), (6, 2), (7, 1), (32, 4), (16, 1), (12, 1), (20, 1)][i]


@pytest.mark.parametrize("dtype", [BF16, FP16])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("lens,new,h,block,window,sinks", [
    ([1], [1], 0, 16, 0, 0), ([1, 2, 127, 128, 129, 257], [1] * 6, 2, 16, 0, 0), ([1000, 31, 33, 640], [1] * 4, 4, 24, 0, 0), ([5000], [1], 1, 2, 0, 0),
    ([777, 3000, 40], [1, 2, 1], 3, 8, 100, 5), ([2500, 1], [1, 1], 4, 64, 129, 0), ([300, 600, 900], [2, 1, 2], 0, 16, 0, 0), ([1234], [1], 5, 32, 0, 0),
    ([1234, 4000], [1, 1], 6, 128, 700, 130), ([500, 9], [4, 3], 1, 16, 0, 0), ([70, 7], [3, 7], 2, 256, 0, 0), ([12000, 100], [1, 1], 0, 16, 3000, 1)])
def test_attention_of_few_rows(dtype, d, lens, new, h, block, window, sinks):
    hq, hkv = heads(h)
    c = Case(dtype, lens, new, hq, hkv, d, block, seed=len(lens) + block)
    want = c.want(window, sinks)
    c.check(c.run(window, sinks, hint=max(new), tail=3), want, few=max(new) * hq // hkv <= 16)
    c.check(c.run(window, sinks, hint=0, lse=False), want)       # without the hint other kernels may serve
    assert kvc.kvc_poll_device_status(c.lay) == (0, 0)


@pytest.mark.parametrize("dtype", [BF16, FP16])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("lens,new,h,block,window,sinks", [
    ([128], [128], 1, 16, 0, 0), ([300, 77, 511], [300, 20, 1], 2, 16, 0, 0), ([1000], [33], 0, 24, 0, 0), ([900, 2000], [900, 100], 4, 64, 0, 0),
    ([700, 1500, 64], [650, 3, 64], 3, 8, 200, 7), ([2049], [257], 5, 2, 0, 0), ([1025, 513], [1025, 40], 1, 128, 100, 0), ([40, 50], [40, 50], 6, 32, 0, 0),
    ([260, 1], [260, 1], 7, 256, 90, 64), ([3000, 17], [18, 17], 0, 16, 1000, 3)])
def test_attention_of_many_rows(dtype, d, lens, new, h, block, window, sinks):
    hq, hkv = heads(h)
    c = Case(dtype, lens, new, hq, hkv, d, block, seed=len(lens) + block)
    want = c.want(window, sinks)
    c.check(c.run(window, sinks, hint=max(new), tail=5), want)
    c.check(c.run(window, sinks, hint=1), want)                  # a hint never changes what is computed
    assert kvc.kvc_poll_device_status(c.lay) == (0, 0)


@pytest.mark.parametrize("block", [1, 3, 5, 48, 200])
def test_block_sizes_that_tiles_are_not_made_of(block):
    c = Case(BF16, [500, 130, 1], [200, 1, 1], 8, 2, 128, block, seed=block)
    want = c.want()
    for hint in (0, 1):
        c.check(c.run(hint=hint), want)


@pytest.mark.parametrize("dtype,d,hq,hkv", [(BF16, 128, 8, 1), (FP16, 64, 6, 2), (BF16, 64, 4, 4), (FP16, 128, 32, 4)])
@pytest.mark.parametrize("rows", ["one", "some", "many"])
def test_attention_over_shared_prefixes(dtype, d, hq, hkv, rows):
    block = 16
    lens = [700, 650, 900, 641, 50, 400, 260]
    new = {"one": [1] * 7, "some": [1, 3, 2, 1, 4, 1, 2], "many": [60, 10, 200, 1, 50, 140, 3]}[rows]
    # two groups, the second's prefix ends inside a block; request 4 belongs to none
    c = Case(dtype, lens, new, hq, hkv, d, block, seed=3, shared=[(0, 4, 40), (5, 7, 16)])
    want = c.want()
    groups = ([0, 4, 5, 7], [640, 0, 250])
    for hint in (max(new), 0):
        c.check(c.run(groups=groups, hint=hint, tail=2), want)
    assert kvc.kvc_poll_device_status(c.lay) == (0, 0)


@pytest.mark.parametrize("hint", [1, 2, 30, 300])
def test_tables_that_name_no_block_and_lengths_that_make_no_sense(hint):
    c = Case(BF16, [300, 200, 90, -4, 0], [1, 2, 30, 1, 2], 4, 2, 128, 16, seed=9)
    c.tables[0, 3] = 10**6
    c.tables[1, 0] = -1
    c.check(c.run(hint=hint), c.want())
    skipped, expired = kvc.kvc_poll_device_status(c.lay)
    assert skipped >= 2 * 2 * 16 and expired == 0
    # a longer length than the table has entries: the keys that are not there are left out
    d = Case(BF16, [64, 100], [1, 1], 4, 2, 64, 16, seed=10)
    d.wide = 3
    d.check(d.run(hint=hint), d.want())
    # more query rows than keys: those before the sequence see nothing
    e = Case(FP16, [3, 40], [9, 50], 4, 2, 64, 16, seed=11)
    e.check(e.run(hint=hint), e.want())


def test_places_that_no_query_sees_may_hold_anything():
    """Steps and offsets of infinity and NaN in slots behind the lengths, in other heads' padding and in unused blocks."""
    for new in ([1, 2], [100, 40]):
        c = Case(BF16, [333, 210], new, 8, 2, 128, 16, seed=4)
        want, got = c.want(100, 3), c.run(100, 3)
        used = torch.zeros(c.nb, c.block, dtype=torch.bool)
        for r, n in enumerate(c.lens):
            for j in range(n):
                if j >= n - new[r] - 99 or j < 3:
                    used[c.tables[r, j // 16], j % 16] = True
        for p in range(2):
            codes, step, offset = [x.clone() for x in c.parts[p]]
            step[~used.cuda()], offset[~used.cuda()] = math.inf, math.nan
            c.pool[1, p] = q4.pack_slabs(codes, step, offset)
        again = c.run(100, 3)
        c.check(again, want)
        assert torch.equal(again[0], got[0]) and torch.equal(again[1], got[1])


@pytest.mark.parametrize("dtype,d,block", [(BF16, 128, 16), (FP16, 64, 24), (FP16, 128, 3), (BF16, 64, 64)])
@pytest.mark.parametrize("new,h", [([1, 1, 1], 0), ([1, 1, 1], 6), ([2, 1, 2], 4), ([9, 1, 5], 1), ([100, 300, 2], 2), ([41, 17, 5], 3)])
@pytest.mark.parametrize("window,sinks", [(0, 0), (130, 3), (1, 0), (64, 70)])
def test_every_row_sees_its_keys_and_no_others(dtype, d, block, new, h, window, sinks):
    """With queries of zeros the log-sum-exp is the logarithm of the number of keys, to 2^-18 of rounding where one key more
    or less is 2^-10; and a query of many times a key's values has that key's value for its result: every row looks for
    a key of its own, the ends of what it sees among them."""
    hq, hkv = heads(h)
    lens = [777, 300, 130]
    c = Case(dtype, lens, new, hq, hkv, d, block, seed=block + h)
    keep = c.q
    c.q = torch.zeros_like(keep)
    rows = [(r, lens[r] - new[r] + i) for r in range(3) for i in range(new[r])]
    seen = [[j for j in range(p + 1) if window == 0 or p - j < window or j < sinks] for _, p in rows]
    count = torch.tensor([len(s) for s in seen], dtype=torch.float64).log().cuda()
    for hint in (max(new), 0):
        lse = c.run(window, sinks, hint=hint)[1]
        assert ((lse.double() - count[:, None]).abs() <= 2.0**-18 + count[:, None] * 2.0**-21).all()
    k, v = (q4.values(*p) for p in c.parts)
    at = torch.empty(c.t, hq, dtype=torch.long)
    for i, s in enumerate(seen):
        ends = [s[0], s[-1], s[len(s) // 2], s[min(sinks, len(s)) - 1 if sinks else 0], s[min(sinks, len(s) - 1)]]
        for x in range(hq):
            j = ends[(i + x) % 5] if x % 2 == 0 else s[(i * 37 + x * 101) % len(s)]
            at[i, x] = c.tables[rows[i][0], j // block] * block + j % block
    head = torch.arange(hq) // (hq // hkv)
    pick = lambda x: x.view(-1, hkv, d)[at.cuda(), head.cuda()]
    c.q = (pick(k) * 20).to(dtype)
    want = pick(v)
    half = torch.finfo(dtype).eps / 2
    # scores: the key's own is about 20 * 1.5^2 * sqrt(d) >= 350, the others are spread by 45 around 0: their weights are nothing.  The value
    # is rounded to the type, and so is the result
    for hint in (max(new), 0):
        out = c.run(window, sinks, hint=hint)[0]
        assert ((out.double() - want).abs() <= 2 * half * want.abs() + 2.0**-20).all()


def test_extreme_scores():
    """Scores of hundreds, of which one key takes all; equal scores; scores near each other far from zero."""
    for factor, shift in ((60.0, 0.0), (0.0, 0.0), (1.0, 40.0)):
        for new in (1, 40):
            c = Case(BF16, [600], [new], 8, 1, 128, 16, seed=6)
            c.q = (c.q.float() * factor + shift).to(BF16)
            c.check(c.run(hint=new), c.want())


@pytest.mark.parametrize("q_power,k_power", [(0, 0), (12, 0), (0, 10), (-6, -9)])
@pytest.mark.parametrize("lens,new,h", [([300, 129, 64], [100, 60, 3], 4), ([40, 33], [40, 33], 6), ([2000], [9], 7)])
def test_keys_of_bf16_keep_eleven_bits(q_power, k_power, lens, new, h):
    """Over many rows a key is rounded to 11 bits whatever the type, and queries and keys may be large or small: half a step
    is 2^-12 of a key, and what is below fp16's normal range is off by 2^-25."""
    hq, hkv = heads(h)
    c = Case(BF16, lens, new, hq, hkv, 128, 16, seed=3)
    c.q *= 2.0**q_power
    for i in (1, 2):
        c.parts[0][i] *= 2.0**k_power
    for p in range(2):
        c.pool[1, p] = q4.pack_slabs(*c.parts[p])
    scale = 2.0 ** (-q_power - k_power) * 128**-0.5
    want = c.want(scale=scale)
    got = c.run(hint=max(new), scale=scale)
    c.check(got, want)
    products = want[3][1] / (2.0**-8 + 136 * 2.0**-23)                 # the largest scale * sum_d |q_d k_d|
    most_q, most_k = c.q.double().abs().max(), q4.values(*c.parts[0]).abs().max()
    slip = products * (2.0**-12 + 136 * 2.0**-23) + scale * 128 * 2.0**-25 * (most_q + most_k)
    assert ((got[1].double() - want[1]).abs() <= slip + 2.0**-18 + want[1].abs() * 2.0**-21).all()


@pytest.mark.parametrize("dtype", [BF16, FP16])
@pytest.mark.parametrize("lens,new,h,window,sinks", [
    ([2, 1, 5], [2, 1, 5], 7, 0, 0), ([100, 128, 3], [1, 6, 2], 7, 0, 0), ([900, 40], [6, 5], 7, 100, 28), ([1000], [4], 6, 1, 0)])
def test_rows_that_see_few_keys_take_them_for_what_they_are(dtype, lens, new, h, window, sinks):
    hq, hkv = heads(h)
    c = Case(dtype, lens, new, hq, hkv, 64, 16, seed=5)
    want = c.want(window, sinks)
    c.check(c.run(window, sinks, hint=max(new), tail=2), want, few=True)


@pytest.mark.parametrize("dtype,new,window,sinks", [(FP16, 30, 0, 0), (FP16, 64, 0, 0), (FP16, 300, 1, 0), (FP16, 300, 20, 44), (BF16, 300, 1, 4), (BF16, 300, 16, 0)])
def test_many_rows_that_see_few_keys(dtype, new, window, sinks):
    c = Case(dtype, [new, 7], [new, 7], 12, 2, 128, 8, seed=6)
    want = c.want(window, sinks)
    c.check(c.run(window, sinks, hint=new, tail=2), want, few=True)


def test_strides_and_layers():
    """Queries and results as parts of wider rows, head-major and token-major."""
    c = Case(FP16, [400, 90], [3, 90], 6, 2, 64, 16, seed=8)
    want = c.want()
    for order in (0, 1):
        wide = torch.full((c.t, 10, 72) if order == 0 else (10, c.t, 72), 4.0, dtype=FP16, device="cuda")
        src = torch.full_like(wide, math.nan)
        view = (lambda x: x[:, 2:8, :64]) if order == 0 else (lambda x: x[2:8, :, :64].transpose(0, 1))
        view(src).copy_(c.q)
        ws = torch.empty(kvc.kvc_attention_q4_workspace_bytes(c.lay, c.t, 2, 6), dtype=torch.uint8, device="cuda")
        kvc.kvc_attention_q4(c.lay, 1, view(src), view(wide), c.tables.cuda()[:, : c.wide], torch.tensor(c.lens, **I32), torch.tensor(c.cu, **I32), ws)
        c.check((view(wide).contiguous(), None), want)
        rest = wide.clone()
        view(rest).fill_(4.0)
        assert (rest == 4).all()


def test_the_same_bits_every_time_and_on_two_streams():
    a = Case(BF16, [5000, 300, 1, 8000], [1, 1, 1, 1], 32, 4, 128, 16, seed=1)
    b = Case(FP16, [700, 900], [700, 100], 8, 2, 64, 16, seed=2)
    first = a.run(), b.run()
    s = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    for _ in range(5):
        got = []
        for c, st in zip((a, b), s):
            with torch.cuda.stream(st):
                out, lse = torch.empty_like(c.q), torch.empty(c.t, c.hq, device="cuda")
                ws = torch.empty(kvc.kvc_attention_q4_workspace_bytes(c.lay, c.t, len(c.lens), c.hq), dtype=torch.uint8, device="cuda")
                got.append((out, lse, ws, c.tables.cuda()[:, : c.wide], torch.tensor(c.lens, **I32), torch.tensor(c.cu, **I32)))
        torch.cuda.synchronize()
        for c, st, (out, lse, ws, tab, lens, cu) in zip((a, b), s, got):
            kvc.kvc_attention_q4(c.lay, 1, c.q, out, tab, lens, cu, ws, lse=lse, stream=st)
        torch.cuda.synchronize()
        for (out, lse, *_), (w_out, w_lse) in zip(got, first):
            assert torch.equal(out, w_out) and torch.equal(lse, w_lse)


# ------------------------------------------------------------------ scale
def test_blocks_past_four_gigabytes_and_long_contexts():
    """A pool whose blocks lie 24 MiB apart, 5 GB a plane; and one of 100,000 keys, lines of many runs."""
    d, hkv, block, nb = 128, 2, 16, 220
    slab = block * hkv * q4.row_bytes(d)
    base = torch.empty(nb * (24 << 20) + slab, dtype=torch.uint8, device="cuda")
    planes = [base, base[slab:]]
    lay = kvc.kvc_layout_create(1, 2, nb, block, hkv, q4.row_bytes(d), 1, block, plane_ptrs=planes, block_stride=24 << 20)
    gen = torch.Generator().manual_seed(3)
    n = 3000
    x = torch.randn(2, n, hkv, d, generator=gen).to(BF16).cuda()
    table = torch.randperm(nb, generator=gen)[: -(-n // block)].to(torch.int32)[None].contiguous()
    j = torch.arange(n)
    slots = (table[0, j // block].long() * block + j % block).cuda()
    kvc.kvc_append_q4(lay, 0, None, x[0], x[1], None, slots, None, None)
    back = torch.zeros_like(x)
    kvc.kvc_read_q4(lay, 0, back[0], back[1], slots)
    want = q4.quantise(x)
    assert torch.equal(back, q4.values(*want).float().to(BF16))
    for new in (1, 70):
        q = torch.randn(new, 8, d, generator=gen).to(BF16).cuda()
        out = torch.zeros_like(q)
        ws = torch.empty(kvc.kvc_attention_q4_workspace_bytes(lay, new, 1, 8), dtype=torch.uint8, device="cuda")
        kvc.kvc_attention_q4(lay, 0, q, out, table.cuda(), torch.tensor([n], **I32), torch.tensor([0, new], **I32), ws)
        parts = [[y[p].view(-1, 1, *y.shape[2:]) for y in want] for p in range(2)]     # one key a block, in order
        w = q4.attention(q, parts, torch.arange(n, dtype=torch.int32)[None], [(0, new)], [n], 1, d ** -0.5)
        assert ((out.double() - w[0]).abs() <= q4.bounds(BF16, *w)[0]).all()
    del base, planes, lay
    torch.cuda.empty_cache()
    c = Case(BF16, [100000, 128, 70000], [1, 1, 1], 8, 1, 128, 16, seed=5)
    c.check(c.run(hint=1), c.want())
    c.check(c.run(hint=20), c.want())
    c.check(c.run(hint=0, window=50000, sinks=2), c.want(50000, 2))


def test_planes_past_64_gigabytes():
    """Blocks 7 GiB apart: a place in the plane is more than 2^32 steps of 16 bytes from its beginning."""
    d, hkv, block, nb, gap = 128, 2, 16, 11, 7 << 30
    slab = block * hkv * q4.row_bytes(d)
    if torch.cuda.mem_get_info()[0] < nb * gap + (4 << 30):
        pytest.skip("needs 81 GB")
    base = torch.empty((nb - 1) * gap + 2 * slab, dtype=torch.uint8, device="cuda")
    lay = kvc.kvc_layout_create(1, 2, nb, block, hkv, q4.row_bytes(d), 1, block, plane_ptrs=[base, base[slab:]], block_stride=gap)
    gen = torch.Generator().manual_seed(8)
    n = nb * block - 5
    x = torch.randn(2, n, hkv, d, generator=gen).to(BF16).cuda()
    table = torch.randperm(nb, generator=gen).to(torch.int32)[None].contiguous()
    j = torch.arange(n)
    slots = (table[0, j // block].long() * block + j % block).cuda()
    kvc.kvc_append_q4(lay, 0, None, x[0], x[1], None, slots, None, None)
    back = torch.zeros_like(x)
    kvc.kvc_read_q4(lay, 0, back[0], back[1], slots)
    want = q4.quantise(x)
    assert torch.equal(back, q4.values(*want).float().to(BF16))
    parts = [[y[p].view(-1, 1, *y.shape[2:]) for y in want] for p in range(2)]         # one key a block, in order
    for new in (1, 70):
        q = torch.randn(new, 8, d, generator=gen).to(BF16).cuda()
        out = torch.zeros_like(q)
        ws = torch.empty(kvc.kvc_attention_q4_workspace_bytes(lay, new, 1, 8), dtype=torch.uint8, device="cuda")
        kvc.kvc_attention_q4(lay, 0, q, out, table.cuda(), torch.tensor([n], **I32), torch.tensor([0, new], **I32), ws)
        w = q4.attention(q, parts, torch.arange(n, dtype=torch.int32)[None], [(0, new)], [n], 1, d ** -0.5)
        assert ((out.double() - w[0]).abs() <= q4.bounds(BF16, *w)[0]).all()
    del base, lay
    torch.cuda.empty_cache()


# ------------------------------------------------------------------ a step of them together
@pytest.mark.parametrize("dtype,d,hq,hkv", [(BF16, 128, 8, 2), (FP16, 64, 6, 6)])
def test_a_step_with_pack_and_unpack(dtype, d, hq, hkv):
    """Prompts, then decoded tokens, by map, append, attention; the blocks leave through pack, come back to other places, and
    attention gives the same bits; the same step replayed from a graph with other lengths."""
    gen = torch.Generator().manual_seed(7)
    block, nb, layers, layer = 16, 60, 3, 1
    slab = block * hkv * q4.row_bytes(d)
    pool = torch.randint(0, 256, (layers, 2, nb, slab), generator=gen, dtype=torch.uint8).cuda()
    lay = kvc.kvc_layout_create_q4(pool, layers, nb, block, hkv, d, 4 * block)
    wide_pool = torch.zeros(layers, 2, nb, block, hkv, d, dtype=dtype, device="cuda")
    wide = kvc.kvc_layout_create_dense(wide_pool, layers, 2, nb, block, hkv, d, 2, 4 * block)
    table = angles(512, d)
    axis = kvc.kvc_pair_axes([d // 2 - 12, 6, 6])
    cap, r = 200, 2
    tables, free = torch.full((r, 14), -1, **I32), torch.randperm(nb, generator=gen).int().cuda()
    ctx, new, total, cu = torch.zeros(r, **I32), torch.zeros(r, **I32), torch.zeros(r, **I32), torch.zeros(r + 1, **I32)
    pos, slots, counts = torch.zeros(cap, **I32), torch.zeros(cap, dtype=torch.int64, device="cuda"), torch.zeros(3, **I32)
    x = torch.zeros(cap, hq + 2 * hkv, d, dtype=dtype, device="cuda")
    q, out, lse = torch.zeros(cap, hq, d, dtype=dtype, device="cuda"), torch.zeros(cap, hq, d, dtype=dtype, device="cuda"), torch.zeros(cap, hq, device="cuda")
    q2 = torch.zeros_like(q)
    ws = torch.empty(kvc.kvc_attention_q4_workspace_bytes(lay, cap, r, hq), dtype=torch.uint8, device="cuda")

    def step():
        kvc.kvc_map_tokens(lay, ctx, new, free, tables, cu, pos, slots, total_lens=total, counts=counts)
        positions = torch.stack([pos, pos // 2, pos % 16])
        kvc.kvc_append_q4(lay, layer, x[:, :hq], x[:, hq:hq + hkv], x[:, hq + hkv:], q, slots, positions, table, pair_axis=axis)
        kvc.kvc_append_axes(wide, layer, x[:, :hq], x[:, hq:hq + hkv], x[:, hq + hkv:], q2, slots, positions, table, axis)
        kvc.kvc_attention_q4(lay, layer, q, out, tables, total, cu, ws, lse=lse)

    def check(what):
        t = int(cu[-1])
        assert torch.equal(q[:t], q2[:t]), what
        parts = [q4.quantise(wide_pool[layer, p]) for p in range(2)]
        rows = [(int(cu[i]), int(cu[i + 1])) for i in range(r)]
        w = q4.attention(q[:t], parts, tables.cpu(), rows, total.tolist(), block, d ** -0.5)
        b_out, b_lse = q4.bounds(dtype, *w)
        assert ((out[:t].double() - w[0]).abs() <= b_out).all(), what
        assert ((lse[:t].double() - w[1]).abs() <= b_lse).all(), what
        assert kvc.kvc_poll_device_status(lay) == (0, 0)

    new.copy_(torch.tensor([150, 37], **I32))
    x.copy_(torch.randn(x.shape, generator=gen).to(dtype))
    step()
    check("prompts")
    free = free[int(counts[1]):].clone()
    ctx.copy_(total)
    new.copy_(torch.tensor([1, 1], **I32))
    x.copy_(torch.randn(x.shape, generator=gen).to(dtype))
    step()
    torch.cuda.synchronize()
    check("decode")
    # out of the pool and back, to other blocks
    t = int(cu[-1])
    first, ids = out[:t].clone(), [tables[i, : -(-int(total[i]) // block)].clone() for i in range(r)]
    staging = [torch.zeros(kvc.kvc_layout_chunk_bytes(lay, len(i)), dtype=torch.uint8, device="cuda") for i in ids]
    for i, s in zip(ids, staging):
        kvc.kvc_pack(lay, i, s)
    spare = [b for b in range(nb) if b not in set(torch.cat(ids).tolist())]
    moved = []
    for i, s in zip(ids, staging):
        to = torch.tensor([spare.pop() for _ in i], **I32)
        kvc.kvc_unpack(lay, s, to)
        moved.append(to)
    other = tables.clone()
    for k, to in enumerate(moved):
        other[k, : len(to)] = to
    pool[:, :, torch.cat(ids).long()] = 255
    kvc.kvc_attention_q4(lay, layer, q, out, other, total, cu, ws, lse=lse)
    torch.cuda.synchronize()
    assert torch.equal(out[:t], first)
    # the tokens' values, to the pool of 16-bit elements: attention there over the same values
    for k, to in enumerate(moved):
        j = torch.arange(int(total[k]), device="cuda")
        at = to.long()[j // block] * block + j % block
        n = len(j)
        kv = torch.zeros(2, n, hkv, d, dtype=dtype, device="cuda")
        kvc.kvc_read_q4(lay, layer, kv[0], kv[1], at)
        kvc.kvc_append(wide, layer, None, kv[0], kv[1], None, at, None, None)
    again = torch.zeros_like(out)
    ws2 = torch.empty(kvc.kvc_attention_workspace_bytes(wide, cap, r, hq), dtype=torch.uint8, device="cuda")
    kvc.kvc_attention(wide, layer, q, again, other, total, cu, ws2)
    flat = [wide_pool[layer, p] for p in range(2)]
    half = torch.finfo(dtype).eps / 2
    # both sides round weights, values and results: twice the bound of one, whose slip holds the keys' rounding
    parts = [q4.quantise(x) for x in flat]
    exact = q4.attention(q[:t], [q4.unpack_slabs(pool[layer, p], hkv, block, d, dtype) for p in range(2)], other.cpu(), [(int(cu[i]), int(cu[i + 1])) for i in range(r)],
                         total.tolist(), block, d ** -0.5)
    assert ((again[:t].double() - out[:t].double()).abs() <= 2 * q4.bounds(dtype, *exact)[0]).all()


@pytest.mark.parametrize("d,dtype", [(128, BF16), (64, FP16)])
def test_a_captured_step_replayed_with_other_lengths(d, dtype):
    gen = torch.Generator().manual_seed(17)
    hq, hkv, block, nb, cap, r = 8, 2, 16, 80, 90, 3
    pool = torch.zeros(1, 2, nb, block * hkv * q4.row_bytes(d), dtype=torch.uint8, device="cuda")
    lay = kvc.kvc_layout_create_q4(pool, 1, nb, block, hkv, d, block)
    table = angles(1024, d)
    tables, free = torch.full((r, 20), -1, **I32), torch.randperm(nb, generator=gen).int().cuda()
    ctx, new, total, cu = (torch.zeros(n, **I32) for n in (r, r, r, r + 1))
    pos, slots = torch.zeros(cap, **I32), torch.zeros(cap, dtype=torch.int64, device="cuda")
    x = torch.zeros(cap, hq + 2 * hkv, d, dtype=dtype, device="cuda")
    q, out = (torch.zeros(cap, hq, d, dtype=dtype, device="cuda") for _ in range(2))
    k_back, v_back = (torch.zeros(cap, hkv, d, dtype=dtype, device="cuda") for _ in range(2))
    ws = torch.empty(kvc.kvc_attention_q4_workspace_bytes(lay, cap, r, hq), dtype=torch.uint8, device="cuda")

    def step(stream=None):
        kvc.kvc_map_tokens(lay, ctx, new, free, tables, cu, pos, slots, total_lens=total, stream=stream)
        kvc.kvc_append_q4(lay, 0, x[:, :hq], x[:, hq:hq + hkv], x[:, hq + hkv:], q, slots, pos, table, stream=stream)
        kvc.kvc_read_q4(lay, 0, k_back, v_back, slots, stream=stream)
        kvc.kvc_attention_q4(lay, 0, q, out, tables, total, cu, ws, stream=stream)

    step()                                   # without tokens: nothing to do, but the handle is ready
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    used, lens = 0, [0] * r
    for new_lens in ([40, 7, 0], [1, 1, 30], [1, 1, 1], [0, 50, 2]):
        ctx.copy_(torch.tensor(lens, **I32))
        new.copy_(torch.tensor(new_lens, **I32))
        need = sum(-(-(a + b) // block) - -(-a // block) for a, b in zip(lens, new_lens))
        free.copy_(torch.roll(free, 0))
        x.copy_(torch.randn(x.shape, generator=gen).to(dtype))
        out.fill_(9)
        graph.replay()
        torch.cuda.synchronize()
        free.copy_(torch.roll(free, -need))  # the next step takes from where this one ended
        used += need
        lens = [a + b for a, b in zip(lens, new_lens)]
        t = sum(new_lens)
        parts = [q4.unpack_slabs(pool[0, p], hkv, block, d, dtype) for p in range(2)]
        rows = [(int(cu[i]), int(cu[i + 1])) for i in range(r)]
        w = q4.attention(q[:t], parts, tables.cpu(), rows, lens, block, d ** -0.5)
        assert ((out[:t].double() - w[0]).abs() <= q4.bounds(dtype, *w)[0]).all()
        assert (out[t:] == 9).all()
        want = q4.values(*q4.quantise(x[:t, hq + hkv:])).float().to(dtype)
        assert torch.equal(v_back[:t], want)
    assert used <= nb and kvc.kvc_poll_device_status(lay) == (0, 0)

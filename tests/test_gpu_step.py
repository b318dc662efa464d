"""The operators of a serving step on a B200 against 64-bit loops: token mapping, norm + rotation + cache
write, attention with window and sinks, attention over shared prefixes, and a run of them together."""
import math

import numpy as np
import pytest
import torch

import step_reference as ref
from paper_2609_11744_b200 import kvc

pytestmark = pytest.mark.gpu
BF16, FP16 = torch.bfloat16, torch.float16


def dev(a, dtype=torch.int32):
    return torch.as_tensor(np.asarray(a), dtype=dtype).cuda()


# ------------------------------------------------------------------ map_tokens
def run_map(ctx, new, free, tables, block, num_blocks, capacity, row=None):
    n = len(ctx)
    wide = tables.shape[1]
    row = row or wide
    big = torch.full((max(n, 1), row), -7, dtype=torch.int32, device="cuda")
    big[:n, :wide] = dev(tables)
    pool = torch.zeros(num_blocks * block * 16, dtype=torch.uint8, device="cuda")
    lay = kvc.kvc_layout_create_dense(pool, 1, 1, num_blocks, block, 1, 8, 2, block)
    o = {k: torch.full((m,), -9, dtype=t, device="cuda") for k, m, t in (
        ("cu_tokens", n + 1, torch.int32), ("positions", capacity, torch.int32), ("slots", capacity, torch.int64),
        ("token_request", capacity, torch.int32), ("total_lens", n, torch.int32), ("counts", 3, torch.int32))}
    kvc.kvc_map_tokens(lay, dev(ctx), dev(new), dev(free), big[:n, :wide], **o)
    torch.cuda.synchronize()
    if row > wide:
        assert (big[:, wide:] == -7).all()
    return big[:n, :wide].cpu().numpy(), {k: v.cpu().numpy() for k, v in o.items()}, kvc.kvc_poll_device_status(lay)[0]


@pytest.mark.parametrize("n,block,kind", [(1, 16, "one"), (1, 1, "some"), (3, 16, "some"), (64, 16, "one"), (65, 24, "mixed"),
                                          (513, 16, "some"), (1001, 8, "mixed"), (700, 64, "none"), (2049, 16, "one")])
@pytest.mark.parametrize("short", [0, 5])
def test_map_tokens(n, block, kind, short):
    rng = np.random.default_rng(n * 31 + block + short)
    ctx = rng.integers(0, 300, n)
    ctx[rng.random(n) < 0.2] = 0
    new = {"one": np.ones(n, int), "some": rng.integers(0, 40, n), "mixed": np.where(rng.random(n) < 0.2, rng.integers(1, 200, n), 1),
           "none": np.zeros(n, int)}[kind]
    held, need = -(-ctx // block), -(-(ctx + new) // block)
    wide = int(need.max()) + 2
    total = int(need.sum()) + 3
    ids = rng.permutation(total).astype(np.int32)
    tables = np.full((n, wide), -5, np.int32)
    at = 0
    for r in range(n):
        tables[r, : held[r]] = ids[at: at + held[r]]
        at += held[r]
    free = ids[at:]
    if short:
        free = free[: max(0, int((need - held).sum()) - short)]
    t = int(new.sum())
    for capacity in (t, t + 37, max(0, t - 3)):
        got_t, got, bad = run_map(ctx, new, free, tables, block, total, capacity, wide + 3)
        w = ref.map_tokens(ctx, new, free, tables, block, wide, total, capacity)
        assert np.array_equal(got_t, w[0])
        for k, x in zip(("cu_tokens", "positions", "slots", "token_request", "total_lens", "counts"), w[1:]):
            assert np.array_equal(got[k], x), k
        assert bad == 0


def test_map_tokens_narrow_tables_bad_entries_and_negative_lengths():
    # row 0 runs out of table entries, row 1 holds an id outside the pool, row 2's lengths are negative
    ctx, new = np.array([30, 5, -4, 0]), np.array([20, 4, -3, 0])
    tables = np.array([[3, 4], [99, 0], [1, 1], [1, 1]], np.int32)
    free = np.array([7, 8, 9], np.int32)
    got_t, got, bad = run_map(ctx, new, free, tables, 16, 12, 24)
    w = ref.map_tokens(ctx, new, free, tables, 16, 2, 12, 24)
    assert np.array_equal(got_t, w[0])
    for k, x in zip(("cu_tokens", "positions", "slots", "token_request", "total_lens", "counts"), w[1:]):
        assert np.array_equal(got[k], x), k
    assert got["counts"].tolist() == [24, 0, 18] and bad == 4   # request 1's four tokens met the bad entry


def test_map_tokens_without_requests_and_with_the_most():
    _, got, _ = run_map([], [], [1], np.zeros((0, 4), np.int32), 16, 4, 6)
    assert got["cu_tokens"].tolist() == [0] and (got["slots"] == -1).all() and got["counts"].tolist() == [0, 0, 0]
    n = kvc.KVC_MAP_MAX_REQUESTS
    ctx, new = np.arange(n) % 19, (np.arange(n) % 3 == 0).astype(int)
    tables = np.arange(n * 2, dtype=np.int32).reshape(n, 2)
    free = np.arange(2 * n, 3 * n, dtype=np.int32)
    got_t, got, _ = run_map(ctx, new, free, tables, 16, 3 * n, int(new.sum()))
    w = ref.map_tokens(ctx, new, free, tables, 16, 2, 3 * n, int(new.sum()))
    assert np.array_equal(got_t, w[0]) and np.array_equal(got["slots"], w[3])


# ------------------------------------------------------------------ append
def make_layout(pool, block, order="dense"):
    """A layout over pool [L][2][NB][B][Hkv][D] (dense), or the same planes given one by one."""
    layers, planes, nb, b, hkv, d = pool.shape
    if order == "planes":
        return kvc.kvc_layout_create(layers, planes, nb, b, hkv, d, 2, b, plane_ptrs=[pool[i, j] for i in range(layers) for j in range(planes)])
    return kvc.kvc_layout_create_dense(pool, layers, planes, nb, b, hkv, d, 2, b)


@pytest.mark.parametrize("dtype", [BF16, FP16])
@pytest.mark.parametrize("t,hq,hkv,d,rot,interleaved,norm,block", [
    (1, 1, 1, 8, 0, False, True, 16), (1, 32, 8, 128, 128, False, True, 16), (3, 4, 4, 64, 64, True, True, 16),
    (67, 12, 4, 64, 32, True, True, 24), (33, 7, 1, 80, 80, False, True, 16), (130, 5, 5, 96, 16, False, False, 8),
    (19, 0, 2, 128, 64, False, True, 16), (700, 28, 4, 128, 128, True, False, 64), (41, 16, 2, 256, 256, False, True, 16),
    (9, 3, 1, 200, 96, True, True, 16), (5, 2, 1, 16, 16, False, True, 1), (2100, 8, 1, 128, 0, False, True, 16)])
def test_append(dtype, t, hq, hkv, d, rot, interleaved, norm, block):
    g = torch.Generator().manual_seed(t + d)
    nb = -(-t // block) + 4
    pool = torch.randn(2, 2, nb, block, hkv, d, generator=g).to(dtype).cuda()
    before = pool.clone()
    lay = make_layout(pool, block, "planes" if t % 2 else "dense")
    # heads in one packed row, with a gap behind it that keeps rows 16-byte aligned
    qkv = torch.randn(t, (hq + 2 * hkv) * d + 8, generator=g).to(dtype).cuda()
    q, k, v = (qkv[:, a * d: b * d].view(t, b - a, d) if b > a else None for a, b in ((0, hq), (hq, hq + hkv), (hq + hkv, hq + 2 * hkv)))
    out = torch.full((t, hq, d), 7.0, dtype=dtype, device="cuda") if hq else None
    slots = torch.randperm(nb * block, generator=g)[:t]
    positions = torch.randint(0, 500, (t,), generator=g, dtype=torch.int32)
    skip, lost, far = slots.new_zeros(t, dtype=torch.bool), 0, 0
    if t > 8:
        slots[3], skip[3] = -1, True
        slots[5], skip[5], lost = nb * block, True, 1
        if rot:
            positions[7], skip[7], far = 500, True, 1
    angle = torch.arange(500.0, dtype=torch.float64)[:, None] * 10000.0 ** (-torch.arange(0, max(rot, 1), 2, dtype=torch.float64) / max(rot, 1))
    table = torch.cat([angle.cos(), angle.sin()], 1).float().cuda() if rot else None
    w = [(1 + 0.2 * torch.randn(d, generator=g)).to(dtype).cuda() if norm else None for _ in range(2)]
    kvc.kvc_append(lay, 1, q, k, v, out, slots.cuda(), positions.cuda() if rot else None, table, q_weight=w[0], k_weight=w[1],
                   eps=1e-5, interleaved=interleaved)
    torch.cuda.synchronize()
    assert kvc.kvc_poll_device_status(lay) == (lost + far, 0)
    keep = ~skip
    safe = torch.where(keep, positions, torch.zeros_like(positions)).cuda()
    half = torch.finfo(dtype).eps / 2

    def check(got, x, weight):
        want = ref.norm_rotate(x, weight, 1e-5, safe, table, rot, interleaved)
        # the rounding to the type, and 32-bit work before it: d + 8 roundings of the sum of squares, halved by the
        # root, and a dozen more, on values of which a rotated pair adds two
        size = want.abs() + ref.norm_rotate(x, weight, 1e-5, safe, None, 0, False).abs().amax(-1, keepdim=True)
        bound = half * want.abs() + (d / 2 + 16) * 2.0**-24 * size + 2.0**-25
        assert ((got.double() - want).abs() <= bound).all()

    if hq:
        check(out[keep], q[keep.cuda()], w[0]) if not rot else None
        full = ref.norm_rotate(q, w[0], 1e-5, safe, table, rot, interleaved)
        size = full.abs() + ref.norm_rotate(q, w[0], 1e-5, safe, None, 0, False).abs().amax(-1, keepdim=True)
        ok = (out.double() - full).abs() <= half * full.abs() + (d / 2 + 16) * 2.0**-24 * size + 2.0**-25
        assert ok[keep.cuda()].all()
        assert (out[skip.cuda()] == 7.0).all()
    full = ref.norm_rotate(k, w[1], 1e-5, safe, table, rot, interleaved)
    size = full.abs() + ref.norm_rotate(k, w[1], 1e-5, safe, None, 0, False).abs().amax(-1, keepdim=True)
    flat = pool.view(2, 2, nb * block, hkv, d)
    sel = keep.cuda()
    got = flat[1, 0][slots.cuda()[sel]]
    assert ((got.double() - full[sel]).abs() <= (half * full.abs() + (d / 2 + 16) * 2.0**-24 * size + 2.0**-25)[sel]).all()
    assert torch.equal(flat[1, 1][slots.cuda()[sel]], v[sel])
    # everything else in the pool is as it was
    rest = torch.ones(nb * block, dtype=torch.bool, device="cuda")
    rest[slots.cuda()[sel]] = False
    was = before.view(2, 2, nb * block, hkv, d)
    assert torch.equal(flat[0], was[0]) and torch.equal(flat[1][:, rest], was[1][:, rest])


def test_append_in_place_and_by_head_strides():
    """Queries rotated in place, and heads laid out [heads][tokens][dim]."""
    t, hq, hkv, d = 21, 4, 2, 64
    g = torch.Generator().manual_seed(5)
    pool = torch.zeros(1, 2, 4, 16, hkv, d, dtype=BF16, device="cuda")
    lay = make_layout(pool, 16)
    q = torch.randn(hq, t, d, generator=g).to(BF16).cuda().transpose(0, 1)
    k = torch.randn(hkv, t, d, generator=g).to(BF16).cuda().transpose(0, 1)
    v = torch.randn(1, 1, d, generator=g).to(BF16).cuda().expand(t, hkv, d)   # one value row for all
    angle = torch.arange(64.0)[:, None] * 0.5 ** torch.arange(32.0)
    table = torch.cat([angle.cos(), angle.sin()], 1).cuda()
    positions, slots = torch.arange(t, dtype=torch.int32).cuda(), torch.arange(t).cuda()
    out = torch.zeros(t, hq, d, dtype=BF16, device="cuda")
    kvc.kvc_append(lay, 0, q, k, v, out, slots, positions, table)
    kvc.kvc_append(lay, 0, q, k, v, q, slots, positions, table)
    assert torch.equal(q, out) and torch.equal(pool[0, 1].view(64, hkv, d)[:t], v)


# ------------------------------------------------------------------ attention
class Batch:
    """Requests with their own blocks in a pool whose every other slot is NaN."""

    def __init__(self, lens, rows, hq, hkv, d, dtype, block, seed=0, share=None, lead=0, tail=3, block_pad=0, scatter=False):
        g = torch.Generator().manual_seed(seed)
        n = len(lens)
        need = [max(1, -(-x // block)) for x in lens]
        nb = sum(need) + 4
        self.wide = max(need) + 2
        slab = block * hkv * d
        self.raw = torch.full((2 * 2 * nb * (slab + block_pad),), math.nan, dtype=dtype, device="cuda")
        self.planes = [self.raw[i * nb * (slab + block_pad):][: nb * (slab + block_pad)].view(nb, slab + block_pad)[:, :slab].view(nb, block, hkv, d)
                       for i in range(4)]
        e = 2
        self.lay = kvc.kvc_layout_create(2, 2, nb, block, hkv, d, e, block, base=self.raw, layer_stride=2 * nb * (slab + block_pad) * e,
                                         plane_stride=nb * (slab + block_pad) * e, block_stride=(slab + block_pad) * e)
        ids = torch.randperm(nb, generator=g).tolist()
        tables = np.full((n, self.wide), nb + 5, np.int32)   # entries behind a request's blocks are nonsense
        self.keys, self.values = [], []
        at = 0
        for r in range(n):
            mine = ids[at: at + need[r]]
            at += need[r]
            k = torch.randn(lens[r], hkv, d, generator=g).to(dtype)
            v = torch.randn(lens[r], hkv, d, generator=g).to(dtype)
            if share is not None and share[r][0] != r:      # the first share[r][1] tokens are those of another request
                first, m = share[r]
                k[:m], v[:m] = self.keys[first][:m], self.values[first][:m]
                if m % block == 0:
                    mine[: m // block] = tables[first, : m // block].tolist()
            self.keys.append(k)
            self.values.append(v)
            tables[r, : need[r]] = mine
            for j in range(lens[r]):
                self.planes[2][mine[j // block], j % block] = k[j].cuda()
                self.planes[3][mine[j // block], j % block] = v[j].cuda()
        self.tables_np = tables
        self.lens, self.rows = lens, []
        for m in rows:
            lo = self.rows[-1][1] if self.rows else lead
            self.rows.append((lo, lo + m))
        t = self.rows[-1][1] + tail
        self.cu = dev([lead] + [b for _, b in self.rows])
        self.tables, self.seq = dev(tables), dev(lens)
        if scatter:      # rows of a wider buffer, heads apart
            q = torch.randn(t, hq + 2, d + 8, generator=g).to(dtype).cuda()
            self.q = q[:, 1: hq + 1, :d]
            self.out = torch.full((hq, t, d), 7.0, dtype=dtype, device="cuda").transpose(0, 1)
        else:
            self.q = torch.randn(t, hq, d, generator=g).to(dtype).cuda()
            self.out = torch.full((t, hq, d), 7.0, dtype=dtype, device="cuda")
        self.lse = torch.full((t, hq), 7.0, device="cuda")
        self.dtype, self.d, self.hq = dtype, d, hq

    def workspace(self, groups=0):
        n = kvc.kvc_attention_workspace_bytes(self.lay, self.q.shape[0], len(self.lens), self.hq, groups)
        return torch.full((n,), 0xFF, dtype=torch.uint8, device="cuda")   # NaN wherever something is read unwritten

    def check(self, window=0, sinks=0, scale=None, bad=0):
        torch.cuda.synchronize()
        skipped, gave_up = kvc.kvc_poll_device_status(self.lay)
        assert (skipped > 0) == (bad > 0) and gave_up == 0
        scale = self.d ** -0.5 if scale is None else scale
        out, lse, weight, slip = ref.attention(self.q, self.keys, self.values, self.rows, self.lens, scale, window, sinks)
        b_out, b_lse = ref.attention_bounds(self.dtype, out, lse, weight, slip)
        a, b = self.rows[0][0], self.rows[-1][1]
        got, got_lse = self.out.double().cpu(), self.lse.double().cpu()
        worst = ((got - out).abs() / b_out)[a:b].max() if b > a else 0.0
        assert not got[a:b].isnan().any() and worst <= 1.0, float(worst)
        empty = lse[a:b] == -math.inf
        assert torch.equal(got_lse[a:b] == -math.inf, empty)
        assert (((got_lse - lse).abs() <= b_lse)[a:b] | empty).all()
        for x in (got, got_lse):
            assert (x[:a] == 7.0).all() and (x[b:] == 7.0).all()


SHAPES = [(4, 1, 64), (8, 2, 128), (5, 5, 64), (7, 1, 128), (16, 1, 64), (40, 2, 128), (32, 1, 64)]
SETS = [  # (lengths, query rows)
    ([1], [1]), ([63], [1]), ([64], [1]), ([65], [1]), ([700], [1]), ([1, 17, 128, 129, 300], [1, 1, 1, 1, 1]),
    ([33, 40, 0, 90], [2, 3, 0, 4]), ([5, 64, 200], [5, 64, 37]), ([300, 9], [130, 9]), ([140], [140]), ([2, 0, 3], [4, 2, 3])]


@pytest.mark.parametrize("lens,rows", SETS)
@pytest.mark.parametrize("hq,hkv,d", SHAPES)
def test_attention(lens, rows, hq, hkv, d):
    dtype = BF16 if (hq + len(lens)) % 2 else FP16
    b = Batch(lens, rows, hq, hkv, d, dtype, block=16, seed=len(lens) + hq)
    kvc.kvc_attention(b.lay, 1, b.q, b.out, b.tables, b.seq, b.cu, b.workspace(), lse=b.lse, max_q_len=max(rows))
    b.check()


@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 1), (7, 3), (64, 0), (65, 64), (100, 130), (1000, 4), (130, 1)])
@pytest.mark.parametrize("lens,rows", [([300], [1]), ([700, 1, 129], [1, 1, 1]), ([200, 90], [130, 5]), ([3, 400], [5, 2]),
                                       ([500], [300])])
def test_attention_window_and_sinks(lens, rows, window, sinks):
    for hq, hkv, d, dtype in ((6, 2, 64, FP16), (8, 1, 128, BF16)):
        b = Batch(lens, rows, hq, hkv, d, dtype, block=16, seed=window)
        kvc.kvc_attention(b.lay, 1, b.q, b.out, b.tables, b.seq, b.cu, b.workspace(), window=window, sinks=sinks, lse=b.lse,
                          max_q_len=max(rows))
        b.check(window, sinks)


@pytest.mark.parametrize("block", [1, 8, 20, 24, 64, 256])
@pytest.mark.parametrize("hint", [0, 1, "real"])
def test_attention_block_sizes_strides_and_hints(block, hint):
    for rows in ([1, 1, 2], [70, 1, 33]):
        b = Batch([257, 31, 90], rows, 8, 2, 64 if block % 8 else 128, BF16, block, seed=block, lead=2, block_pad=8, scatter=True)
        kvc.kvc_attention(b.lay, 1, b.q, b.out, b.tables, b.seq, b.cu, b.workspace(), scale=0.3, lse=b.lse,
                          max_q_len=max(rows) if hint == "real" else hint)
        b.check(scale=0.3)


def test_attention_keys_that_are_not_there():
    """Entries outside the pool, and lengths past the table's end: those keys are not seen."""
    for rows in ([1, 1], [40, 3]):
        b = Batch([200, 100], rows, 4, 2, 128, BF16, 16, seed=3)
        b.tables[0, 3] = -1
        b.tables[1, 0] = 10 ** 9
        for k in (b.keys, b.values):
            k[0] = torch.cat([k[0][:48], k[0][64:]])
            k[1] = k[1][16:]
        kvc.kvc_attention(b.lay, 1, b.q, b.out, b.tables, b.seq, b.cu, b.workspace(), lse=b.lse, max_q_len=max(rows))
        # the keys behind the hole move up in the reference, and so do the positions
        b.lens = [184, 84]
        b.check(bad=1)


def test_attention_table_shorter_than_the_length():
    b = Batch([100, 64], [1, 1], 4, 2, 64, BF16, 16, seed=4)
    few = b.tables[:, :4].contiguous()
    kvc.kvc_attention(b.lay, 1, b.q, b.out, few, b.seq, b.cu, b.workspace(), lse=b.lse, max_q_len=1)
    b.keys[0], b.values[0], b.lens = b.keys[0][:64], b.values[0][:64], [64, 64]
    b.check()


def test_attention_block_offsets_past_32_bits():
    """Blocks a gigabyte apart: 64-bit offsets on every path."""
    block, hkv, d, nb = 16, 2, 128, 5
    stride = 1 << 30
    raw = torch.zeros(nb * stride + (1 << 20), dtype=torch.uint8, device="cuda")
    slab = block * hkv * d * 2
    lay = kvc.kvc_layout_create(1, 2, nb, block, hkv, d, 2, block, base=raw, layer_stride=nb * stride, plane_stride=slab, block_stride=stride)
    g = torch.Generator().manual_seed(1)
    for rows in (1, 64):
        t = 64
        k, v = (torch.randn(t, hkv, d, generator=g).to(BF16) for _ in range(2))
        q = torch.randn(rows, 8, d, generator=g).to(BF16).cuda()
        order = [4, 0, 3, 2]
        slots = torch.tensor([order[j // block] * block + j % block for j in range(t)]).cuda()
        kvc.kvc_append(lay, 0, None, k.cuda(), v.cuda(), None, slots, None, None)
        out, lse = torch.zeros_like(q), torch.zeros(rows, 8, device="cuda")
        ws = torch.empty(kvc.kvc_attention_workspace_bytes(lay, rows, 1, 8), dtype=torch.uint8, device="cuda")
        kvc.kvc_attention(lay, 0, q, out, dev([order]), dev([t]), dev([0, rows]), ws, lse=lse, max_q_len=rows)
        want, wl, weight, slip = ref.attention(q, [k], [v], [(0, rows)], [t], d ** -0.5)
        b_out, _ = ref.attention_bounds(BF16, want, wl, weight, slip)
        assert ((out.double().cpu() - want).abs() <= b_out).all()


def test_attention_large_scores_do_not_overflow():
    """Scores of several hundred: only their differences reach the exponential."""
    for rows in (1, 50):
        b = Batch([150], [rows], 4, 2, 64, BF16, 16, seed=8)
        kvc.kvc_attention(b.lay, 1, b.q, b.out, b.tables, b.seq, b.cu, b.workspace(), scale=16.0, lse=b.lse, max_q_len=rows)
        b.check(scale=16.0)


# ------------------------------------------------------------------ shared prefixes
@pytest.mark.parametrize("lens,rows,groups,prefix", [
    ([40, 33], [1, 1], [0, 2], [32]), ([200, 177, 160, 161], [1, 1, 1, 1], [0, 4], [160]),
    ([90, 80, 300, 301, 65], [1, 2, 1, 3, 1], [0, 2, 4, 5], [64, 256, 0]), ([100, 100, 50], [1, 1, 1], [0, 2], [96]),
    ([70, 90], [1, 1], [0, 2], [37]), ([300, 280, 290], [20, 1, 70], [0, 3], [208]), ([50, 60], [10, 30], [0, 2], [48]),
    ([64, 64], [1, 1], [0, 2], [64]), ([500] * 20, [1] * 20, [0, 20], [480])])
@pytest.mark.parametrize("hq,hkv,d", [(8, 2, 128), (4, 4, 64), (12, 1, 64)])
def test_attention_shared(lens, rows, groups, prefix, hq, hkv, d):
    share = []
    for r in range(len(lens)):
        g = max([i for i in range(len(prefix)) if groups[i] <= r] or [0])
        share.append((groups[g], prefix[g]) if groups[g] <= r < groups[g + 1] else (r, 0))
    dtype = BF16 if d == 128 else FP16
    b = Batch(lens, rows, hq, hkv, d, dtype, 16, seed=len(lens), share=share, lead=1)
    kvc.kvc_attention_shared(b.lay, 1, b.q, b.out, b.tables, b.seq, b.cu, dev(groups), dev(prefix), b.workspace(len(prefix)),
                             lse=b.lse, max_q_len=max(rows))
    b.check()


# ------------------------------------------------------------------ conventions
def test_same_bits_again_on_another_stream_and_in_a_graph():
    b = Batch([900, 20, 333], [1, 1, 1], 8, 2, 128, BF16, 16, seed=11)
    ws = b.workspace()
    call = lambda **kw: kvc.kvc_attention(b.lay, 1, b.q, b.out, b.tables, b.seq, b.cu, ws, lse=b.lse, max_q_len=1, **kw)
    call()
    torch.cuda.synchronize()
    first = b.out.clone()
    side = torch.cuda.Stream()
    b.out.fill_(7.0)
    side.wait_stream(torch.cuda.current_stream())
    call(stream=side)
    side.synchronize()
    assert torch.equal(first, b.out)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    b.out.fill_(7.0)
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(first, b.out)
    # lengths are read when the graph runs
    b.seq.copy_(dev([700, 20, 16]))
    for k in (b.keys, b.values):
        k[0], k[2] = k[0][:700], k[2][:16]
    b.lens = [700, 20, 16]
    graph.replay()
    b.check()


def test_tensors_are_refused_before_a_launch():
    b = Batch([40], [1], 4, 2, 64, BF16, 16)
    ws = b.workspace()
    n = kvc.kvc_layout_launch_count(b.lay)

    def refused(err, **kw):
        a = dict(q=b.q, out=b.out, block_tables=b.tables, seq_lens=b.seq, cu_tokens=b.cu, workspace=ws)
        a.update(kw)
        with pytest.raises(err):
            kvc.kvc_attention(b.lay, 1, **a)

    refused(TypeError, q=b.q.float())
    refused(TypeError, out=b.out.half())
    refused(ValueError, out=b.out[:, :2])
    refused(ValueError, q=b.q.cpu())
    refused(TypeError, block_tables=b.tables.long())
    refused(ValueError, seq_lens=b.seq.cpu())
    refused(ValueError, cu_tokens=b.cu[:1])
    refused(ValueError, lse=torch.zeros(1, device="cuda"))
    refused(kvc.KvcError, workspace=ws[: 1024])
    refused(kvc.KvcError, workspace=torch.empty(ws.numel() + 256, dtype=torch.uint8, device="cuda")[16:])
    refused(ValueError, workspace=torch.empty(ws.numel(), dtype=torch.uint8))
    refused(kvc.KvcError, scale=0.0)
    q = torch.zeros(4, 4, 68, dtype=BF16, device="cuda")[..., :64]
    refused(kvc.KvcError, q=q, out=torch.zeros(4, 4, 64, dtype=BF16, device="cuda"))
    assert kvc.kvc_layout_launch_count(b.lay) == n


def test_a_step_from_lengths_to_a_packed_chunk_and_back():
    """Two steps of three requests: map, append, attend; then the cache is packed with the device-resident
    tables, unpacked into other blocks, and attention over those gives the same bits."""
    hq, hkv, d, block, nb = 8, 2, 128, 16, 64
    g = torch.Generator().manual_seed(2)
    pool = torch.full((2, 2, nb, block, hkv, d), math.nan, dtype=BF16, device="cuda")
    lay = make_layout(pool, block)
    n, wide, cap = 3, 12, 128
    tables = torch.full((n, wide), -1, dtype=torch.int32, device="cuda")
    free = torch.randperm(nb, generator=g).int().cuda()
    ctx = torch.zeros(n, dtype=torch.int32, device="cuda")
    angle = torch.arange(256.0)[:, None] * 0.9 ** torch.arange(64.0)
    cs = torch.cat([angle.cos(), angle.sin()], 1).cuda()
    w = (1 + 0.1 * torch.randn(d, generator=g)).to(BF16).cuda()
    keys, values, used = [[] for _ in range(n)], [[] for _ in range(n)], 0
    for new in ([37, 5, 64], [1, 1, 1], [1, 0, 20]):
        cu, pos = torch.zeros(n + 1, dtype=torch.int32, device="cuda"), torch.zeros(cap, dtype=torch.int32, device="cuda")
        slots, total = torch.zeros(cap, dtype=torch.int64, device="cuda"), torch.zeros(n, dtype=torch.int32, device="cuda")
        counts = torch.zeros(3, dtype=torch.int32, device="cuda")
        kvc.kvc_map_tokens(lay, ctx, dev(new), free[used:], tables, cu, pos, slots, total_lens=total, counts=counts)
        x = torch.randn(cap, hq + 2 * hkv, d, generator=g).to(BF16).cuda()
        q = torch.full((cap, hq, d), 7.0, dtype=BF16, device="cuda")
        kvc.kvc_append(lay, 1, x[:, :hq], x[:, hq: hq + hkv], x[:, hq + hkv:], q, slots, pos, cs, q_weight=w, k_weight=w)
        out, lse = torch.full_like(q, 7.0), torch.full((cap, hq), 7.0, device="cuda")
        ws = torch.empty(kvc.kvc_attention_workspace_bytes(lay, cap, n, hq), dtype=torch.uint8, device="cuda")
        kvc.kvc_attention(lay, 1, q, out, tables, total, cu, ws, lse=lse, max_q_len=max(new))
        torch.cuda.synchronize()
        c = cu.tolist()
        assert c[-1] == sum(new) and counts.tolist()[2] == 0 and (q[c[-1]:] == 7.0).all() and (out[c[-1]:] == 7.0).all()
        used += int(counts[1])
        flat = pool[1].view(2, nb * block, hkv, d)
        for r in range(n):
            s = slots[c[r]: c[r + 1]]
            keys[r].append(flat[0][s].cpu())
            values[r].append(x[c[r]: c[r + 1], hq + hkv:].cpu())
        ks, vs = [torch.cat(k) for k in keys], [torch.cat(v) for v in values]
        rows = [(c[r], c[r + 1]) for r in range(n)]
        want, wl, weight, slip = ref.attention(q, ks, vs, rows, total.tolist(), d ** -0.5)
        b_out, b_lse = ref.attention_bounds(BF16, want, wl, weight, slip)
        m = c[-1]
        assert ((out.double().cpu() - want).abs() <= b_out)[:m].all() and ((lse.double().cpu() - wl).abs() <= b_lse)[:m].all()
        ctx.copy_(total)
    moved = torch.full_like(tables, -1)
    spare = free[used:]
    for r in range(n):
        m = -(-int(total[r]) // block)
        slot = torch.empty(kvc.kvc_layout_chunk_bytes(lay, m), dtype=torch.uint8, device="cuda")
        kvc.kvc_pack(lay, tables[r, :m].contiguous(), slot)
        moved[r, :m] = spare[r * 9: r * 9 + m]
        kvc.kvc_unpack(lay, slot, moved[r, :m].contiguous())
    again, lse2 = torch.full_like(out, 7.0), torch.full_like(lse, 7.0)
    kvc.kvc_attention(lay, 1, q, again, moved, total, cu, ws, lse=lse2, max_q_len=20)
    assert torch.equal(again, out) and torch.equal(lse2, lse)
    assert kvc.kvc_poll_device_status(lay) == (0, 0)


def test_attention_pairs_of_one_and_two_row_tiles_in_any_order():
    """Requests whose queries fill one row tile or two, and keys of odd and even numbers of tiles, one after
    the other in the same blocks."""
    rng = np.random.default_rng(5)
    for hq, hkv, d in ((8, 2, 128), (4, 4, 64)):
        lens = rng.integers(1, 1400, 24).tolist()
        rows = [min(x, int(rng.choice([1, 20, 33, 64, 70, 130, 200]))) for x in lens]
        b = Batch(lens, rows, hq, hkv, d, BF16, 16, seed=hq)
        for _ in range(3):
            kvc.kvc_attention(b.lay, 1, b.q, b.out, b.tables, b.seq, b.cu, b.workspace(), lse=b.lse, max_q_len=max(rows))
        b.check()


def test_attention_scores_that_rise_along_the_keys():
    """Keys whose scores grow: the running maximum moves at every tile, and sums are rescaled each time."""
    for rows, hq in ((1, 4), (60, 4), (200, 4)):
        b = Batch([900], [rows], hq, 2, 64, BF16, 16, seed=4)
        grow = torch.linspace(0.0, 40.0, 900)[:, None, None]
        k = (b.keys[0].float() * 0.1 + grow).to(BF16)
        b.q.copy_(b.q.abs())
        b.keys[0] = k
        for j in range(900):
            b.planes[2][b.tables_np[0, j // 16], j % 16] = k[j].cuda()
        kvc.kvc_attention(b.lay, 1, b.q, b.out, b.tables, b.seq, b.cu, b.workspace(), lse=b.lse, max_q_len=rows)
        b.check()


def test_append_with_an_unaligned_angle_table():
    """A cos/sin table at an address that no vector load may use, against the same table aligned."""
    t, hq, hkv, d = 40, 6, 2, 128
    g = torch.Generator().manual_seed(6)
    q, k, v = (torch.randn(t, h, d, generator=g).to(BF16).cuda() for h in (hq, hkv, hkv))
    positions, slots = torch.randint(0, 90, (t,), generator=g, dtype=torch.int32).cuda(), torch.arange(t).cuda()
    raw = torch.randn(90 * 64 + 1, generator=g).cuda()
    got = []
    for table in (raw[1:].view(90, 64), raw[1:].clone().view(90, 64)):
        for interleaved in (False, True):
            pool = torch.zeros(1, 2, 4, 16, hkv, d, dtype=BF16, device="cuda")
            out = torch.zeros_like(q)
            kvc.kvc_append(make_layout(pool, 16), 0, q, k, v, out, slots, positions, table, interleaved=interleaved)
            got.append((out, pool))
    for i in range(2):
        assert torch.equal(got[i][0], got[i + 2][0]) and torch.equal(got[i][1], got[i + 2][1])


def test_attention_window_and_sinks_at_their_limits():
    b = Batch([300, 40], [70, 1], 4, 2, 64, BF16, 16, seed=9)
    for rows in ([70, 1],):
        kvc.kvc_attention(b.lay, 1, b.q, b.out, b.tables, b.seq, b.cu, b.workspace(), window=1 << 30, sinks=1 << 30, lse=b.lse,
                          max_q_len=max(rows))
        b.check()
        kvc.kvc_attention(b.lay, 1, b.q, b.out, b.tables, b.seq, b.cu, b.workspace(), window=1 << 30, lse=b.lse, max_q_len=1)
        b.check()


def test_lengths_that_contradict_one_another_stay_inside_the_buffers():
    """Token rows that descend or overlap, lengths past the table, groups out of order: whatever comes out, nothing
    outside the buffers is touched, no wait gives up, and a sound call afterwards is right."""
    g = torch.Generator().manual_seed(12)
    for hint in (1, 64):
        b = Batch([200, 90, 150], [3, 2, 40], 8, 2, 128, BF16, 16, seed=21, lead=1)
        t = b.q.shape[0]
        frame = torch.full((t + 8, 8, 128), 5.0, dtype=BF16, device="cuda")
        ws = b.workspace(2)
        guard = torch.full((ws.numel() + 4096,), 0x5A, dtype=torch.uint8, device="cuda")
        space = guard[: ws.numel()]
        for cu in ([0, 46, 0, 46], [46, 0, 46, 0], [-5, 1000, 3, 2], [7, 7, 7, 7], [0, 2 ** 31 - 1, 1, 40]):
            for lens in ([200, 90, 150], [2 ** 31 - 1, -3, 10 ** 6], [0, 0, 0]):
                kvc.kvc_attention(b.lay, 1, b.q, frame[4: t + 4], b.tables, dev(lens), dev(cu), space, lse=b.lse, max_q_len=hint)
                for groups, prefix in (([0, 2, 3], [64, 32]), ([3, 1, 0], [10 ** 9, -1]), ([-7, 99, 2], [17, 300])):
                    kvc.kvc_attention_shared(b.lay, 1, b.q, frame[4: t + 4], b.tables, dev(lens), dev(cu), dev(groups), dev(prefix),
                                             space, lse=b.lse, max_q_len=hint)
        torch.cuda.synchronize()
        assert (frame[:4] == 5.0).all() and (frame[t + 4:] == 5.0).all() and (guard[ws.numel():] == 0x5A).all()
        assert kvc.kvc_poll_device_status(b.lay)[1] == 0
        b.lse.fill_(7.0)
        kvc.kvc_attention(b.lay, 1, b.q, b.out, b.tables, b.seq, b.cu, space, lse=b.lse, max_q_len=40)
        b.check()


def test_a_copy_that_does_not_wait_for_copies_waits_for_a_step():
    """pdl = 3: chunks packed right behind kvc_append hold what it wrote."""
    hkv, d, block, nb = 8, 128, 16, 512
    pool = torch.zeros(1, 2, nb, block, hkv, d, dtype=BF16, device="cuda")
    lay = make_layout(pool, block)
    kvc.kvc_layout_set_tuning(lay, pdl=3)
    t = nb * block
    slots = torch.arange(t).cuda()
    ids = torch.arange(nb, dtype=torch.int32).cuda()
    chunks = torch.empty(nb // 64, kvc.kvc_layout_chunk_bytes(lay, 64), dtype=torch.uint8, device="cuda")
    x = [torch.full((t, hkv, d), float(i + 1), dtype=BF16, device="cuda") for i in range(2)]
    torch.cuda.synchronize()
    for i in range(20):
        kvc.kvc_append(lay, 0, None, x[i % 2], x[i % 2], None, slots, None, None)
        for c in range(nb // 64):
            kvc.kvc_pack(lay, ids[c * 64: (c + 1) * 64], chunks[c])
        torch.cuda.synchronize()
        assert (chunks.view(BF16) == float(i % 2 + 1)).all()


def test_a_whole_step_replayed_from_a_graph_with_other_lengths():
    """Map, append, attention and attention over a shared prefix captured once, replayed with fewer and more tokens
    than at capture: lengths are read when the graph runs, and rows behind the last token are left as they were."""
    hq, hkv, d, block, nb, n, cap = 8, 2, 64, 16, 256, 3, 192
    g = torch.Generator().manual_seed(3)
    pool = torch.full((1, 2, nb, block, hkv, d), math.nan, dtype=BF16, device="cuda")
    lay = make_layout(pool, block)
    wide = 40
    tables, free = torch.full((n, wide), -1, dtype=torch.int32, device="cuda"), torch.randperm(nb, generator=g).int().cuda()
    ctx, new = dev([0, 0, 0]), dev([60, 3, 100])
    cu, pos = torch.zeros(n + 1, dtype=torch.int32, device="cuda"), torch.zeros(cap, dtype=torch.int32, device="cuda")
    slots, total = torch.zeros(cap, dtype=torch.int64, device="cuda"), torch.zeros(n, dtype=torch.int32, device="cuda")
    counts = torch.zeros(3, dtype=torch.int32, device="cuda")
    x = torch.randn(cap, hq + 2 * hkv, d, generator=g).to(BF16).cuda()
    q, out, again = (torch.zeros(cap, hq, d, dtype=BF16, device="cuda") for _ in range(3))
    ws = torch.empty(kvc.kvc_attention_workspace_bytes(lay, cap, n, hq, 1), dtype=torch.uint8, device="cuda")
    groups, prefix = dev([0, 1]), dev([48])   # the first request alone: its first blocks count as a prefix

    def step():
        kvc.kvc_map_tokens(lay, ctx, new, free, tables, cu, pos, slots, total_lens=total, counts=counts)
        kvc.kvc_append(lay, 0, x[:, :hq], x[:, hq: hq + hkv], x[:, hq + hkv:], q, slots, None, None)
        kvc.kvc_attention(lay, 0, q, out, tables, total, cu, ws, max_q_len=cap)
        kvc.kvc_attention_shared(lay, 0, q, again, tables, total, cu, groups, prefix, ws, max_q_len=cap)

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    held = [[], [], []]
    taken = 0
    for lens in ([60, 3, 100], [1, 0, 1], [70, 90, 2], [1, 1, 1]):
        new.copy_(dev(lens))
        x.copy_(torch.randn(x.shape, generator=g).to(BF16))
        for t in (q, out, again):
            t.fill_(7.0)
        graph.replay()
        torch.cuda.synchronize()
        c = cu.tolist()
        m = c[-1]
        for r in range(n):
            held[r].append((x[c[r]: c[r + 1], hq: hq + hkv].cpu(), x[c[r]: c[r + 1], hq + hkv:].cpu()))
        keys, values = ([torch.cat([a[i] for a in h]) for h in held] for i in range(2))
        want, wl, weight, slip = ref.attention(q, keys, values, [(c[r], c[r + 1]) for r in range(n)], total.tolist(), d ** -0.5)
        bound, _ = ref.attention_bounds(BF16, want, wl, weight, slip)
        for got in (out, again):
            assert ((got.double().cpu() - want).abs() <= bound)[:m].all() and (got[m:] == 7.0).all()
        assert (q[m:] == 7.0).all() and torch.equal(q[:m], x[:m, :hq])
        ctx.copy_(total)
        taken = int(counts[1])
        free.copy_(torch.roll(free, -taken))
    assert kvc.kvc_poll_device_status(lay) == (0, 0)


def test_calls_on_two_streams_at_once():
    """The same handle, two streams, workspaces of their own: the bits of either alone."""
    sets = [Batch([1900, 40, 700], [1, 1, 1], 8, 2, 128, BF16, 16, seed=31), Batch([900, 300], [200, 70], 8, 2, 128, BF16, 16, seed=32)]
    lay = sets[0].lay
    calls = []
    for b, hint in zip(sets, (1, 200)):
        ws = b.workspace()
        calls.append(lambda s, b=b, ws=ws, hint=hint: kvc.kvc_attention(b.lay, 1, b.q, b.out, b.tables, b.seq, b.cu, ws, lse=b.lse,
                                                                       max_q_len=hint, stream=s))
    alone = []
    for b, call in zip(sets, calls):
        call(None)
        torch.cuda.synchronize()
        alone.append((b.out.clone(), b.lse.clone()))
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for _ in range(30):
        for s, call in zip(streams, calls):
            call(s)
    torch.cuda.synchronize()
    for b, (o, l) in zip(sets, alone):
        assert torch.equal(b.out, o) and torch.equal(b.lse, l)
        b.check()
    assert kvc.kvc_poll_device_status(lay) == (0, 0)


@pytest.mark.parametrize("rows", [1, 3, 70])
@pytest.mark.parametrize("window,sinks", [(100, 0), (129, 5), (33, 64)])
def test_attention_does_not_read_what_no_window_reaches(rows, window, sinks):
    """Keys and values behind every window and all sinks are gone: their slots hold NaN, and the blocks that
    held nothing else have no entry in the table."""
    for hq, hkv, d in ((8, 1, 128), (12, 4, 64)):
        b = Batch([700], [rows], hq, hkv, d, BF16 if d == 128 else FP16, 16, seed=window)
        first = 700 - rows + 1 - window       # the first key that some window reaches
        for j in range(sinks, first):
            for plane in b.planes[2:]:
                plane[b.tables_np[0, j // 16], j % 16] = math.nan
        for block in range(-(-sinks // 16), first // 16):
            b.tables[0, block] = -1
        kvc.kvc_attention(b.lay, 1, b.q, b.out, b.tables, b.seq, b.cu, b.workspace(), window=window, sinks=sinks, lse=b.lse,
                          max_q_len=rows)
        b.check(window, sinks)


@pytest.mark.parametrize("rows", [[1, 1, 1], [30, 1, 70]])
def test_attention_shared_reads_the_prefix_through_the_first_request_only(rows):
    """The other requests' table entries for the shared blocks may be missing."""
    for hq, hkv, d in ((8, 2, 128), (12, 1, 64)):
        prefix = 176
        b = Batch([300, 290, 280], rows, hq, hkv, d, BF16, 16, seed=3, share=[(0, prefix)] * 3)
        b.tables[1:, : prefix // 16] = -1
        kvc.kvc_attention_shared(b.lay, 1, b.q, b.out, b.tables, b.seq, b.cu, dev([0, 3]), dev([prefix]), b.workspace(1), lse=b.lse,
                                 max_q_len=max(rows))
        b.check()

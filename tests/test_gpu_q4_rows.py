"""Attention over a pool held in 4 bits on a B200, row by row against bounds of each row's own keys: queries and keys of
any size, rows that see few keys, and ordinary calls by either kernel."""
import pytest
import torch

import q4_reference as q4
import q4_row_bounds as bounds
from paper_2609_11744_b200 import kvc
from test_gpu_q4 import BF16, FP16, Case, heads

pytestmark = pytest.mark.gpu


def store(c):
    for p in range(2):
        c.pool[1, p] = q4.pack_slabs(*c.parts[p])


def keys_times(c, power):
    """power: a whole number, or one a key [block, token]."""
    f = torch.exp2(torch.as_tensor(power, dtype=torch.float32)).to("cuda")
    for i in (1, 2):
        x = c.parts[0][i]
        c.parts[0][i] = (x.float() * (f[..., None, None] if f.dim() else f)).to(x.dtype)
    store(c)


@pytest.mark.parametrize("dtype", [BF16, FP16])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("lens,new,h,block,window,sinks", [
    ([1, 2, 127, 129, 700], [1] * 5, 2, 16, 0, 0), ([3000, 40], [2, 1], 3, 8, 100, 5), ([500, 9], [4, 3], 1, 16, 0, 0), ([900], [1], 7, 24, 64, 70),
    ([300, 77, 511], [300, 20, 1], 2, 16, 0, 0), ([900, 2000], [900, 100], 4, 64, 0, 0), ([700, 1500, 64], [650, 3, 64], 3, 8, 200, 7), ([2049], [257], 5, 2, 0, 0)])
def test_ordinary_calls(dtype, d, lens, new, h, block, window, sinks):
    hq, hkv = heads(h)
    c = Case(dtype, lens, new, hq, hkv, d, block, seed=len(lens) + block, extra=300 // block + 1)
    want = bounds.attention(c, window, sinks)
    few = max(new) * hq // hkv <= 16
    bounds.check(c, c.run(window, sinks, hint=max(new)), want, "few" if few else "many")
    bounds.check(c, c.run(window, sinks, hint=1 if not few else 0), want, "any")


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


@pytest.mark.parametrize("dtype,k_power", [(BF16, -40), (BF16, -24), (BF16, -10), (BF16, 18), (BF16, 40), (FP16, -10), (FP16, -16), (FP16, 9)])
@pytest.mark.parametrize("d,lens,new,h,block", [(64, [333], [1], 0, 16), (128, [900, 70], [2, 1], 0, 24)])
def test_keys_of_any_size(dtype, k_power, d, lens, new, h, block):
    hq, hkv = heads(h)
    c = Case(dtype, lens, new, hq, hkv, d, block, seed=3, extra=300 // block + 1)
    keys_times(c, k_power)
    scale = 2.0**-k_power * d**-0.5
    bounds.check(c, c.run(hint=max(new), scale=scale), bounds.attention(c, scale=scale), "few")


@pytest.mark.parametrize("dtype", [BF16, FP16])
@pytest.mark.parametrize("k_power", [-20, -14, -8, -4, 4, 9, 12])
@pytest.mark.parametrize("d,lens,new,h,block", [(128, [300, 129, 64], [100, 60, 3], 4, 16), (64, [600, 40], [600, 40], 2, 24), (128, [900], [9], 7, 128)])
def test_keys_of_the_sizes_that_many_rows_take(dtype, k_power, d, lens, new, h, block):
    """Up to 65504, and small ones off by 2^-25; whatever the hint."""
    hq, hkv = heads(h)
    c = Case(dtype, lens, new, hq, hkv, d, block, seed=3, extra=300 // block + 1)
    keys_times(c, k_power if dtype is BF16 else min(k_power, 11))
    scale = 2.0**-k_power * d**-0.5
    want = bounds.attention(c, scale=scale)
    bounds.check(c, c.run(hint=max(new), scale=scale), want, "many")
    bounds.check(c, c.run(hint=1, scale=scale), want, "any")


@pytest.mark.parametrize("new", [1, 20, 300])
@pytest.mark.parametrize("window,sinks", [(0, 0), (90, 3)])
def test_neighbouring_keys_of_different_sizes(new, window, sinks):
    c = Case(BF16, [400], [new], 8, 2, 128, 16, seed=4, extra=9)
    n = c.nb * c.block
    # stretches of 32 keys of one size, and keys that differ from their neighbours
    keys_times(c, ((torch.arange(n) // 32 * 13) % 30 - 20).view(c.nb, c.block))
    keys_times(c, (torch.arange(n) * 5 % 7 - 3).view(c.nb, c.block))
    for scale in (128**-0.5 * 2.0**-2, 128**-0.5 * 2.0**-9):
        want = bounds.attention(c, window, sinks, scale)
        bounds.check(c, c.run(window, sinks, hint=new, scale=scale), want, "few" if new == 1 else "many")


def test_a_key_that_is_not_finite_leaves_rows_that_do_not_see_it_alone():
    """Keys of infinity and NaN in the middle of a prompt: rows before them, and behind a window, are what they were."""
    for dtype in (BF16, FP16):
        c = Case(dtype, [300], [300], 4, 1, 128, 16, seed=6, extra=9)
        want, got = bounds.attention(c, 40, 0), c.run(40, 0, hint=300)
        j = 150
        at = (int(c.tables[0, j // 16]), j % 16)
        for what in (float("inf"), float("nan")):
            c.parts[0][1][at], c.parts[0][2][at] = what, what
            store(c)
            again = c.run(40, 0, hint=300)
            keep = torch.ones(300, dtype=torch.bool)
            keep[j: j + 40] = False
            assert torch.isfinite(again[0][keep.cuda()]).all() and torch.isfinite(again[1][keep.cuda()]).all()
            assert not torch.isfinite(again[1][~keep.cuda()]).any()
            for a, b in zip(again, got):
                a[~keep.cuda()] = b[~keep.cuda()]
            bounds.check(c, again, want, "many")


@pytest.mark.parametrize("dtype", [BF16, FP16])
@pytest.mark.parametrize("extra", [0, 500])
@pytest.mark.parametrize("d,lens,new,h,window,sinks", [
    (128, [1, 2, 5, 700, 64, 65], [1, 2, 5, 700, 64, 65], 2, 0, 0), (64, [3, 900, 40], [3, 200, 40], 4, 0, 0), (128, [400], [400], 5, 64, 0), (64, [400, 300], [400, 290], 2, 20, 44),
    (128, [700, 31], [300, 31], 4, 1, 3), (128, [50, 30, 3], [9, 9, 3], 4, 0, 0), (64, [300, 200], [300, 10], 1, 33, 0), (128, [129], [129], 6, 3, 61)])
def test_rows_that_see_few_keys(dtype, extra, d, lens, new, h, window, sinks):
    """Whatever the width of the table, the other requests of the call and the hint."""
    hq, hkv = heads(h)
    c = Case(dtype, lens, new, hq, hkv, d, 16, seed=5, extra=extra)
    want = bounds.attention(c, window, sinks)
    for hint in (max(new), 0, 1):
        bounds.check(c, c.run(window, sinks, hint=hint), want, "any")
    assert kvc.kvc_poll_device_status(c.lay) == (0, 0)


@pytest.mark.parametrize("dtype", [BF16, FP16])
@pytest.mark.parametrize("prefix", [16, 48, 64, 200])
def test_rows_that_see_few_keys_behind_a_shared_prefix(dtype, prefix):
    lens = [prefix + 3, prefix + 1, prefix + 12, 9]
    new = [3, 1, 12, 9]
    for h in (2, 4, 5):
        hq, hkv = heads(h)
        c = Case(dtype, lens, new, hq, hkv, 128, 16, seed=7, extra=100, shared=[(0, 3, -(-prefix // 16))])
        want = bounds.attention(c)
        for hint in (12, 0):
            bounds.check(c, c.run(groups=([0, 3], [prefix]), hint=hint), want, "any")


def test_one_graph_of_rows_of_all_kinds():
    """A call captured once and replayed with other queries, keys and lengths: no power of two and no choice is kept."""
    c = Case(BF16, [300, 500], [40, 30], 8, 2, 128, 16, seed=8, extra=9)
    dev = [torch.tensor(x, dtype=torch.int32, device="cuda") for x in (c.lens, c.cu)]
    q, out, lse = c.q.clone(), torch.zeros_like(c.q), torch.zeros(c.t, c.hq, device="cuda")
    tables = c.tables.cuda()[:, : c.wide]
    ws = torch.empty(kvc.kvc_attention_q4_workspace_bytes(c.lay, c.t, 2, c.hq), dtype=torch.uint8, device="cuda")
    kvc.kvc_attention_q4(c.lay, 1, q, out, tables, *dev, ws, lse=lse, max_q_len=40)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        kvc.kvc_attention_q4(c.lay, 1, q, out, tables, *dev, ws, lse=lse, max_q_len=40)
    parts = [[x.clone() for x in p] for p in c.parts]
    for q_power, k_power, lens in ((0, 0, [300, 500]), (20, -8, [40, 500]), (-30, 12, [300, 31]), (0, 0, [300, 500])):
        c.parts = [[x.clone() for x in p] for p in parts]
        keys_times(c, k_power)
        q.copy_((c.q.float() * 2.0**q_power).to(BF16))
        dev[0].copy_(torch.tensor(lens, dtype=torch.int32))
        graph.replay()
        torch.cuda.synchronize()
        keep, c.q, c.lens = c.q, q, lens
        want = bounds.attention(c)
        bounds.check(c, (out, lse), want, "many")
        c.q = keep

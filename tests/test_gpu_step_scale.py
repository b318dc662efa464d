"""Attention at lengths and numbers of requests that leave the small cases' arithmetic: rows joined from more than 32
parts, lines of units past 2^20, prompts and drafted tokens behind long loaded contexts."""
import math

import pytest
import torch

import step_reference as ref
from paper_2609_11744_b200 import kvc
from test_gpu_step import BF16, FP16, dev, make_layout

pytestmark = pytest.mark.gpu


class Pool:
    """One sequence of `keys` keys in scattered blocks; requests are prefixes of it, through tables of their own."""

    def __init__(self, keys, hkv, d, dtype, block, seed):
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.need = -(-keys // block)
        nb = self.need + 3
        self.pool = torch.full((1, 2, nb, block, hkv, d), math.nan, dtype=dtype, device="cuda")
        self.ids = torch.randperm(nb, generator=g, device="cuda")[: self.need].int()
        self.kv = torch.randn(2, keys, hkv, d, generator=g, device="cuda").to(dtype)
        at = self.ids.long()[torch.arange(keys, device="cuda") // block] * block + torch.arange(keys, device="cuda") % block
        self.pool[0].view(2, nb * block, hkv, d)[:, at] = self.kv
        self.lay, self.g = make_layout(self.pool, block), g
        self.dtype, self.d, self.hkv = dtype, d, hkv

    def queries(self, t, hq):
        q = torch.randn(t, hq, self.d, generator=self.g, device="cuda")
        q[:, 1::2] *= 6.0   # the odd heads' weights gather on a few keys, so that what is left out or weighed twice shows
        q[t // 2:, 0] *= 6.0
        q = q.to(self.dtype)
        return q, torch.full_like(q, 7.0), torch.full((t, hq), 7.0, device="cuda")

    def check(self, q, out, lse, pos):
        """Against 64-bit arithmetic; pos: the position of every row.

        Beside what the small cases' bounds count, sums of n terms in 32 bits, added one after the other in the worst
        case: sums of weights take at most n / 4 additions in one place and products n / 16 (a matrix instruction
        takes 16 keys), half a step each, and 64 more for joins."""
        t, hq, d = q.shape
        keys = int(pos.max()) + 1
        g, scale = hq // self.hkv, d ** -0.5
        half = torch.finfo(self.dtype).eps / 2
        worst = worst_lse = 0.0
        for h in range(self.hkv):
            k, v = self.kv[0, :keys, h].double(), self.kv[1, :keys, h].double()
            top_k = float(k.abs().max())
            step = max(1, (1 << 26) // keys // g)
            for a in range(0, t, step):
                x = q[a: a + step, h * g: (h + 1) * g].double()
                p = pos[a: a + step]
                s = torch.einsum("tgd,kd->tgk", x, k) * scale
                s.masked_fill_((torch.arange(keys, device="cuda") > p[:, None])[:, None], -math.inf)
                z = torch.logsumexp(s, -1)
                w = torch.exp(s - z[..., None])
                want, size = w @ v, w @ v.abs()
                slip = float((x.abs().sum(-1) * top_k).max()) * scale * (d + 4) * 2.0**-24
                sums = (keys / 4 + 64) * 2.0**-24
                b_out, b_lse = ref.attention_bounds(self.dtype, want, z, size, slip)
                b_out = b_out + size * (sums + (keys / 16 + 64) * 2.0**-24)
                worst = max(worst, float(((out[a: a + step, h * g: (h + 1) * g].double() - want).abs() / b_out).max()))
                worst_lse = max(worst_lse, float(((lse[a: a + step, h * g: (h + 1) * g].double() - z).abs() / (b_lse + sums)).max()))
        assert worst <= 1.0 and worst_lse <= 1.0, (worst, worst_lse)
        assert kvc.kvc_poll_device_status(self.lay) == (0, 0)


def positions(lens, rows):
    return torch.cat([torch.arange(n - m, n) for n, m in zip(lens, rows)]).cuda()


def attend(p, lens, rows, hq, groups=None, repeat=1):
    n, t = len(lens), sum(rows)
    tables = p.ids[None].expand(n, p.need).contiguous()
    cu = [0]
    for m in rows:
        cu.append(cu[-1] + m)
    q, out, lse = p.queries(t, hq)
    ws = torch.full((kvc.kvc_attention_workspace_bytes(p.lay, t, n, hq, len(groups[1]) if groups else 0),), 0xFF, dtype=torch.uint8, device="cuda")
    first, args = None, (p.lay, 0, q, out, tables, dev(lens), dev(cu))
    for _ in range(repeat):
        if groups:
            kvc.kvc_attention_shared(*args, dev(groups[0]), dev(groups[1]), ws, lse=lse, max_q_len=max(rows))
        else:
            kvc.kvc_attention(*args, ws, lse=lse, max_q_len=max(rows))
        if repeat > 1:
            first = first or (out.clone(), lse.clone())
            assert torch.equal(first[0], out) and torch.equal(first[1], lse)
    p.check(q, out, lse, positions(lens, rows))


@pytest.mark.parametrize("rows", [1, 2, 5, 40])
@pytest.mark.parametrize("hq,hkv,d", [(8, 1, 128), (6, 2, 64)])
def test_few_tokens_behind_80000(rows, hq, hkv, d):
    """A pair's keys are cut between more than 32 blocks, and its rows joined from as many parts."""
    attend(Pool(80000, hkv, d, BF16, 16, rows), [79999], [rows], hq)


@pytest.mark.parametrize("dtype,keys", [(BF16, 32000), (FP16, 8000)])
def test_prompts_behind_loaded_contexts(dtype, keys):
    """New tokens behind cached ones, without a window: rows of one row tile and of several, with decode tokens beside them."""
    attend(Pool(keys, 2, 128, dtype, 16, 5), [keys - 5, keys, 700, keys // 2], [256, 1, 300, 33], 8)


def test_one_row_tile_over_32000_keys_repeats():
    attend(Pool(32000, 1, 128, BF16, 16, 6), [32000], [16], 8, repeat=1000)


@pytest.mark.parametrize("rows", [1, 20])
def test_a_line_of_more_than_2_to_the_20_units(rows):
    """1024 requests with 8 KV heads: at 8192 keys (tiles of 64, and one for the pair) or 16384 (tiles of 128, and three)
    the line is longer than 2^20, where the places of its cuts are computed in 64 bits."""
    keys = 8192 if rows == 1 else 16384
    lens = [keys - r % 5 for r in range(1024)]
    assert 1024 * 8 * (keys // 64 + 1 if rows == 1 else keys // 128 + 3) >= 1 << 20
    attend(Pool(keys, 8, 64, BF16, 16, 7), lens, [rows] * 1024, 8)


@pytest.mark.parametrize("rows", [1, 3])
@pytest.mark.parametrize("hq,hkv", [(4, 1), (16, 2)])
def test_shared_prefix_of_more_than_32_parts(rows, hq, hkv):
    n = 40
    lens = [32000 + 7 * r + rows for r in range(n)]
    attend(Pool(max(lens), hkv, 128, BF16, 16, 8), lens, [rows] * n, hq, groups=([0, n - 2], [32000]))

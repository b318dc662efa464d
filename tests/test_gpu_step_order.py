"""What a step's calls owe to the order of things: the two halves of a row in the attention tiles, copies and steps
on one stream and on several, results that repeat."""
import pytest
import torch

from paper_2609_11744_b200 import kvc
from test_gpu_step import BF16, FP16, Batch

pytestmark = pytest.mark.gpu


def set_keys(b, r, k):
    """Replaces the keys of request r of a batch (one copy)."""
    b.keys[r] = k.to(b.dtype)
    j = torch.arange(k.shape[0])
    block = b.planes[2].shape[1]
    ids = torch.as_tensor(b.tables_np[r]).long()[j // block]
    b.planes[2][ids.cuda(), (j % block).cuda()] = b.keys[r].cuda()


@pytest.mark.parametrize("hq,hkv,d,dtype", [(8, 1, 128, BF16), (4, 2, 64, FP16)])
def test_halves_of_a_tile_share_one_maximum(hq, hkv, d, dtype):
    """One row tile over many key tiles, where the two halves of a tile's keys have maxima far apart, in turns: both
    have to weigh by the larger one.  Repeated, with the same bits."""
    rows, n = 120 // (hq // hkv), 5000
    b = Batch([n], [rows], hq, hkv, d, dtype, 16, seed=7)
    j = torch.arange(n)
    far = ((j // 64 + j // 128) % 2).float() * 6.0 + (j // 128).float() * 0.05   # the upper half of even tiles, the lower of odd ones
    b.q.copy_(b.q.abs())
    set_keys(b, 0, b.keys[0].float() * 0.2 + far[:, None, None] * d ** -0.5)
    ws = b.workspace()
    first = None
    for _ in range(200):
        kvc.kvc_attention(b.lay, 1, b.q, b.out, b.tables, b.seq, b.cu, ws, lse=b.lse, max_q_len=rows)
        if first is None:
            first = b.out.clone(), b.lse.clone()
        assert torch.equal(first[0], b.out) and torch.equal(first[1], b.lse)
    b.check()


@pytest.mark.parametrize("rows,d,dtype", [(30, 128, BF16), (100, 64, FP16), (120, 128, BF16)])
def test_results_rescaled_at_every_tile_repeat(rows, d, dtype):
    """Maxima that grow by more than 2^8 from key tile to key tile, so that both halves of a row rescale their columns
    of the result again and again while products wait: right, and the same bits each time."""
    n = 3000
    b = Batch([n, 1500], [rows, rows], 4, 1, d, dtype, 16, seed=8)
    b.q.copy_(b.q.abs())
    for r, m in enumerate((n, 1500)):
        grow = (torch.arange(m) // 128).float() * (7.0 if r else 9.0) / (0.8 * d ** 0.5)
        set_keys(b, r, b.keys[r].float() * 0.1 + grow[:, None, None])
    ws = b.workspace()
    first = None
    for _ in range(200):
        kvc.kvc_attention(b.lay, 1, b.q, b.out, b.tables, b.seq, b.cu, ws, lse=b.lse, max_q_len=rows)
        if first is None:
            first = b.out.clone(), b.lse.clone()
        assert torch.equal(first[0], b.out) and torch.equal(first[1], b.lse)
    b.check()

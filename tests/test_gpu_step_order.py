"""What a step's calls owe to the order of things: the two halves of a row in the attention tiles, copies and steps
on one stream and on several, results that repeat."""
import pytest
import torch

from paper_2609_11744_b200 import kvc
from test_gpu_step import BF16, FP16, Batch, dev, make_layout

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


def copies_then_step(nb=2048, hkv=8, d=128, block=16):
    pool = torch.zeros(1, 2, nb, block, hkv, d, dtype=BF16, device="cuda")
    lay = make_layout(pool, block)
    kvc.kvc_layout_set_tuning(lay, pdl=3, slot_memory=1)
    return pool, lay, torch.arange(nb, dtype=torch.int32).cuda()


@pytest.mark.parametrize("graphed", [False, True])
@pytest.mark.parametrize("rows", [1, 24])
def test_attention_behind_copies_that_do_not_wait_reads_what_all_of_them_wrote(graphed, rows):
    """pdl = 3: a large unpack, two of a single block, then attention over the large one's blocks.  All keys are alike, so
    the result is the value that every block holds, exactly."""
    nb, hkv, d, block, n = 2048, 8, 128, 16, 64
    pool, lay, ids = copies_then_step(nb, hkv, d, block)
    big = kvc.kvc_layout_chunk_bytes(lay, nb - 2)
    chunk = torch.empty(big, dtype=torch.uint8, device="cuda")
    small = torch.zeros(2, kvc.kvc_layout_chunk_bytes(lay, 1), dtype=torch.uint8, device="cuda")
    tables = torch.arange(n * 31, dtype=torch.int32).view(n, 31).cuda()
    q = torch.ones(n * rows, hkv, d, dtype=BF16, device="cuda")
    out = torch.empty_like(q)
    lens, cu = dev([31 * block] * n), dev([i * rows for i in range(n + 1)])
    ws = torch.empty(kvc.kvc_attention_workspace_bytes(lay, n * rows, n, hkv), dtype=torch.uint8, device="cuda")

    def call():
        kvc.kvc_unpack(lay, chunk, ids[: nb - 2])
        kvc.kvc_unpack(lay, small[0], ids[nb - 2: nb - 1])
        kvc.kvc_unpack(lay, small[1], ids[nb - 1:])
        kvc.kvc_attention(lay, 0, q, out, tables, lens, cu, ws, max_q_len=rows)

    call()
    torch.cuda.synchronize()
    if graphed:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            call()
    for i in range(20):
        chunk.view(BF16).fill_(float(i % 3 + 1))
        torch.cuda.synchronize()
        graph.replay() if graphed else call()
        torch.cuda.synchronize()
        assert (out == float(i % 3 + 1)).all(), i
    assert kvc.kvc_poll_device_status(lay) == (0, 0)


@pytest.mark.parametrize("graphed", [False, True])
def test_append_behind_copies_that_do_not_wait_leaves_them_what_they_read(graphed):
    """pdl = 3: a large pack and one of a single block, then an append into the large one's blocks."""
    nb, hkv, d, block = 2048, 8, 128, 16
    pool, lay, ids = copies_then_step(nb, hkv, d, block)
    chunk = torch.empty(kvc.kvc_layout_chunk_bytes(lay, nb - 1), dtype=torch.uint8, device="cuda")
    small = torch.empty(kvc.kvc_layout_chunk_bytes(lay, 1), dtype=torch.uint8, device="cuda")
    t = (nb - 1) * block
    slots = torch.arange(t).cuda()
    x = torch.empty(t, hkv, d, dtype=BF16, device="cuda")

    def call():
        kvc.kvc_pack(lay, ids[: nb - 1], chunk)
        kvc.kvc_pack(lay, ids[nb - 1:], small)
        kvc.kvc_append(lay, 0, None, x, x, None, slots, None, None)

    call()
    torch.cuda.synchronize()
    if graphed:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            call()
    for i in range(20):
        x.fill_(float(i + 1))
        pool.fill_(float(i))
        chunk.fill_(0xFF)
        torch.cuda.synchronize()
        graph.replay() if graphed else call()
        torch.cuda.synchronize()
        assert (chunk.view(BF16) == float(i)).all(), i
        assert (pool.view(2, nb, -1)[:, : nb - 1] == float(i + 1)).all(), i
    assert kvc.kvc_poll_device_status(lay) == (0, 0)


@pytest.mark.parametrize("other_handle", [False, True])
def test_copies_on_another_stream_do_not_make_the_next_copy_forget_a_step(other_handle):
    """pdl = 3: kvc_append on stream A, a copy on stream B, then a pack on A of what was appended, through the same
    handle or another one on the same pool."""
    nb, hkv, d, block = 1024, 8, 128, 16
    pool, lay, ids = copies_then_step(nb, hkv, d, block)
    packer = lay
    if other_handle:
        packer = make_layout(pool, block)
        kvc.kvc_layout_set_tuning(packer, pdl=3, slot_memory=1)
    side = torch.zeros(kvc.kvc_layout_chunk_bytes(lay, 1), dtype=torch.uint8, device="cuda")
    chunk = torch.empty(8, kvc.kvc_layout_chunk_bytes(lay, nb // 8), dtype=torch.uint8, device="cuda")
    slots = torch.arange((nb - 1) * block).cuda()
    x = torch.empty((nb - 1) * block, hkv, d, dtype=BF16, device="cuda")
    streams = torch.cuda.Stream(), torch.cuda.Stream()
    for i in range(30):
        x.fill_(float(i % 5 + 1))
        torch.cuda.synchronize()
        kvc.kvc_append(lay, 0, None, x, x, None, slots, None, None, stream=streams[0])
        kvc.kvc_pack(lay, ids[nb - 1:], side, stream=streams[1])   # a block that nothing is appended to
        for c in range(8):
            kvc.kvc_pack(packer, ids[c * (nb // 8): (c + 1) * (nb // 8)], chunk[c], stream=streams[0])
        torch.cuda.synchronize()
        got = chunk.view(BF16).view(8, 2, nb // 8, -1).transpose(1, 2).reshape(nb, -1)
        assert (got[: nb - 1] == float(i % 5 + 1)).all() and (got[nb - 1] == 0.0).all(), i
    assert kvc.kvc_poll_device_status(lay) == (0, 0)


def test_copies_captured_behind_a_step_wait_for_it():
    """pdl = 3: kvc_append and packs of what was appended in one graph; a capture takes nothing from the next copy outside it."""
    nb, hkv, d, block = 1024, 8, 128, 16
    pool, lay, ids = copies_then_step(nb, hkv, d, block)
    chunk = torch.empty(8, kvc.kvc_layout_chunk_bytes(lay, nb // 8), dtype=torch.uint8, device="cuda")
    slots = torch.arange(nb * block).cuda()
    x = torch.empty(nb * block, hkv, d, dtype=BF16, device="cuda")

    def packs():
        for c in range(8):
            kvc.kvc_pack(lay, ids[c * (nb // 8): (c + 1) * (nb // 8)], chunk[c])

    def step():
        kvc.kvc_append(lay, 0, None, x, x, None, slots, None, None)

    step()
    packs()
    torch.cuda.synchronize()
    both = torch.cuda.CUDAGraph()
    with torch.cuda.graph(both):
        step()
        packs()
    for i in range(20):
        x.fill_(float(i + 1))
        torch.cuda.synchronize()
        if i % 2:
            both.replay()
        else:
            step()
            if i % 4:
                packs()
            else:
                with torch.cuda.graph(torch.cuda.CUDAGraph()):   # captured, not run, between the step and the copies
                    packs()
                packs()
        torch.cuda.synchronize()
        assert (chunk.view(BF16) == float(i + 1)).all(), i
    assert kvc.kvc_poll_device_status(lay) == (0, 0)

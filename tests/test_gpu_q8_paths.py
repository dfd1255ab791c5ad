"""Branches of fa_q8_attention and fa_q8_step that need many pairs of row and KV head, or many query columns: ragged batches cut as one line of units, steps in
it, and what is not finite, not there or behind a row's end in the kernel for chunks of queries."""
import math

import pytest
import torch

from paper_2506_11886_b200 import fa
from tests import q8_reference as ref
from tests.test_gpu_q8 import DT, attend_and_check, check_cache, make, rand

pytestmark = pytest.mark.gpu


def filled(lens, dtype, fmt, **kw):
    """A cache whose rows hold `lens` tokens of their own, and the tokens."""
    lay, cache = make(B=len(lens), dtype=dtype, fmt=fmt, **kw)
    H, d, most = lay.n_kv_heads, lay.head_dim, max(lens)
    K, V = rand((len(lens), most, H, d), dtype, 1), rand((len(lens), most, H, d), dtype, 2)
    fa.fa_q8_write(lay, cache, K, V, torch.tensor(lens, dtype=torch.int32, device="cuda"))
    rows = ref.Rows(len(lens), H, d, lay.block, fmt, DT[dtype][0])
    for b, n in enumerate(lens):
        rows.push(b, K[b, :n], V[b, :n])
    return lay, cache, rows


# ---- more pairs than CTAs -----------------------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype,fmt,Hq,H,d,block,n_q", [
    ("bf16", "int8", 32, 32, 128, 32, 1),        # 320 pairs with tokens on 296 CTAs
    ("bf16", "e4m3", 96, 48, 64, 16, 1),
    ("bf16", "int8", 48, 16, 64, 64, 5),         # two column tiles to a CTA: 160 pairs on 148
    ("bf16", "e4m3", 16, 16, 256, 16, 1),
    ("f32", "int8", 32, 32, 64, 32, 1),
    ("f32", "e4m3", 16, 16, 128, 16, 11),
    ("bf16", "int8", 4, 2, 64, 16, 31)])         # 4 tiles of 16 columns of 2 heads: 80 pairs, cut into parts
def test_ragged_rows_in_a_line(dtype, fmt, Hq, H, d, block, n_q):
    """Rows of many lengths, empty ones at both ends and side by side; the line's parts end inside rows, blocks and tails."""
    lens = [0, 300, 1, 0, 0, 129, 15, 16, 17, 64, 257, 33, 500, 0]
    lay, cache, rows = filled(lens, dtype, fmt, Hq=Hq, H=H, d=d, block=block, nb=512 // block)
    out, _ = attend_and_check(lay, cache, rows, rand((len(lens), n_q, Hq, d), dtype, 3), dtype)
    for b, n in enumerate(lens):
        assert n or (out[b] == 0).all()


def test_more_than_32_ragged_rows_in_a_line():
    lens = [(53 * b) % 97 if b % 5 else 0 for b in range(70)]
    lay, cache, rows = filled(lens, "bf16", "int8", Hq=8, H=8, d=64, block=16, nb=6)
    attend_and_check(lay, cache, rows, rand((70, 1, 8, 64), "bf16", 3), "bf16")


@pytest.mark.parametrize("dtype,fmt,d,block,B,H,G", [("bf16", "int8", 128, 32, 12, 32, 1), ("bf16", "e4m3", 64, 16, 40, 8, 2), ("f32", "int8", 64, 16, 12, 16, 1),
                                                     ("bf16", "e4m3", 256, 64, 6, 32, 1), ("bf16", "int8", 64, 16, 12, 16, 12)])
def test_steps_in_a_line(dtype, fmt, d, block, B, H, G):
    """Steps of ragged rows over the ends of blocks; rows that are full (with blocks of 64 the third one after its first step) and one that needs a page that is
    not there attend to what they hold."""
    lens = [(37 * b + 13 * (b % 3)) % 100 for b in range(B)]
    lens[0], lens[1], lens[2], lens[3], lens[4] = 0, block - 2, 2 * block - 1, 128, block - 1
    lay, cache, rows = filled(lens, dtype, fmt, Hq=G * H, H=H, d=d, block=block, nb=128 // block)
    good = cache.block_table.clone()
    cache.block_table[4, 0] = lay.n_pages
    ws = fa.new_q8_workspace(lay)
    for i in range(4):
        q, k, v = rand((B, G * H, d), dtype, 10 + i), rand((B, H, d), dtype, 20 + i), rand((B, H, d), dtype, 30 + i)
        out = torch.full_like(q, math.nan)
        fa.fa_q8_step(lay, cache, q, k, v, out, ws)
        assert fa.fa_q8_poll_status(cache) in (fa.FA_ERR_CAPACITY, fa.FA_ERR_INDEX)
        assert (ws[:4096] == 0).all()
        for b in range(B):
            if b != 4 and rows.k[b].shape[0] < 128:
                rows.push(b, k[b:b + 1], v[b:b + 1])
        assert cache.state[:, 0].tolist() == [x.shape[0] for x in rows.k]
        got = out.cpu().double()
        for b in range(B):
            for h in range(0, H, 1 if i == 3 else 5):
                want, tol = ref.attention(rows.held("k", b, h), rows.held("v", b, h), q[b, None, h * G:(h + 1) * G].cpu().double(), 1, lay.softmax_scale, DT[dtype][0])
                assert ((got[b, None, h * G:(h + 1) * G] - want).abs() <= tol).all(), (i, b, h)
    cache.block_table.copy_(good)
    check_cache(lay, cache, rows, fmt)


# ---- many query columns -------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
def test_chunks_and_what_is_behind_a_row(fmt):
    """NaN in the tails behind the rows' last tokens, in pages and scales of nobody, a block table that is none past the rows' blocks: bit for bit the same.
    Then a tail and a block that are not finite: NaN for the queries that see them, the others bit for bit the same."""
    B, Hq, H, d, block, n_q = 2, 8, 2, 128, 32, 40
    lay, cache = make(B=B, Hq=Hq, H=H, d=d, block=block, nb=6, fmt=fmt)
    K, V = rand((B, 100, H, d), "bf16", 1), rand((B, 100, H, d), "bf16", 2)
    lens = torch.tensor([100, 70], dtype=torch.int32, device="cuda")
    fa.fa_q8_write(lay, cache, K, V, lens)
    q, ws = rand((B, n_q, Hq, d), "bf16", 3), fa.new_q8_workspace(lay, n_q)
    out, dirty = torch.empty_like(q), torch.empty_like(q)
    fa.fa_q8_attention(lay, cache, q, out, ws)
    used = torch.zeros(lay.n_pages, dtype=torch.bool, device="cuda")
    for b, n in enumerate((100, 70)):
        used[cache.block_table[b, :n // block].long()] = True
        for t in (cache.k_tail, cache.v_tail):
            t[b, :, n % block:] = float("nan")
        cache.block_table[b, n // block:] = 1 << 30
    for side in ("k", "v"):
        getattr(cache, side + "_pages").view(torch.uint8)[~used] = 0x7f
        getattr(cache, side + "_scale")[~used] = float("nan")
    ws[4096:].fill_(255)
    fa.fa_q8_attention(lay, cache, q, dirty, ws)
    assert torch.equal(out, dirty) and torch.isfinite(out.float()).all() and fa.fa_q8_poll_status(cache) == fa.FA_OK
    for bad in (float("inf"), float("nan")):
        for side in (K, V):
            keep = side.clone()
            side[0, 97, 0, 5], side[1, 40, 0, 7] = bad, -bad            # in the tail (tokens 96 .. 99) and in block 1 (32 .. 63)
            other = make(B=B, Hq=Hq, H=H, d=d, block=block, nb=6, fmt=fmt)[1]
            fa.fa_q8_write(lay, other, K, V, lens)
            fa.fa_q8_attention(lay, other, q, dirty, ws)
            assert fa.fa_q8_poll_status(other) == fa.FA_OK
            # query i of row 0 sees tokens 0 .. 60 + i, of row 1 0 .. 30 + i; the other head none of it
            for b, first in ((0, 36), (1, 2)):
                assert torch.equal(dirty[b, :first], out[b, :first]) and torch.equal(dirty[b, :, 4:], out[b, :, 4:])
                assert torch.isnan(dirty[b, first:, :4].float()).all()
            side.copy_(keep)


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
def test_chunks_and_pages_out_of_range(fmt):
    """Blocks without a page are left out and reported: single ones of 16 tokens, and all of the 128 that are taken at a time."""
    Hq, H, d, block, n, n_q = 4, 1, 64, 16, 400, 20
    lay, cache, rows = filled([n], "bf16", fmt, Hq=Hq, H=H, d=d, block=block, nb=26)
    gone = [1, 4] + list(range(8, 16)) + [24]
    for i in gone:
        cache.block_table[0, i] = (-1, lay.n_pages, -2 ** 31, 2 ** 31 - 1)[i % 4]
    q = rand((1, n_q, Hq, d), "bf16", 3)
    out, ws = torch.full_like(q, math.nan), fa.new_q8_workspace(lay, n_q)
    fa.fa_q8_attention(lay, cache, q, out, ws)
    assert fa.fa_q8_poll_status(cache) == fa.FA_ERR_INDEX
    k, v = rows.held("k", 0, 0), rows.held("v", 0, 0)
    for i in range(n_q):
        keep = [t for t in range(n - n_q + i + 1) if t // block not in gone]
        want, tol = ref.attention(k[keep], v[keep], q[0, i:i + 1].cpu().double(), 1, lay.softmax_scale, torch.bfloat16)
        assert ((out[0, i].cpu().double() - want[0]).abs() <= tol[0]).all(), i


def test_chunks_of_blocks_of_very_different_scale():
    """V blocks and a tail from 1e-30 to 1e30 and back, K blocks from 1e-6 on; a part of the queries sees a part of them only."""
    Hq, H, d, block, n, n_q = 4, 1, 64, 16, 16 * 12 + 9, 90
    for order in (1, -1):
        f, fk = 10.0 ** (order * torch.linspace(-30, 30, 13)), 10.0 ** torch.linspace(-6, 0, 13)
        lay, cache = make(Hq=Hq, H=H, d=d, block=block, nb=13)
        K = (rand((1, n, H, d), "bf16", 1).float().cpu() * fk.repeat_interleave(block)[None, :n, None, None]).bfloat16().cuda()
        V = (rand((1, n, H, d), "bf16", 2).float().cpu() * f.repeat_interleave(block)[None, :n, None, None]).bfloat16().cuda()
        fa.fa_q8_write(lay, cache, K, V)
        rows = ref.Rows(1, H, d, block, "int8", torch.bfloat16)
        rows.push(0, K[0], V[0])
        attend_and_check(lay, cache, rows, rand((1, n_q, Hq, d), "bf16", 3), "bf16")


def test_captured_appends_chunks_and_reads():
    """A graph of an append, the attention of the chunk and a read, replayed while the rows grow; bit for bit what the eager calls give."""
    B, Hq, H, d, block, n = 2, 8, 2, 128, 16, 24
    made = [make(B=B, Hq=Hq, H=H, d=d, block=block, nb=10) for _ in range(2)]
    K, V, q = rand((B, n, H, d), "bf16", 1), rand((B, n, H, d), "bf16", 2), rand((B, n, Hq, d), "bf16", 3)
    count = torch.tensor([n, n - 5], dtype=torch.int32, device="cuda")
    outs = [[torch.zeros_like(q), torch.zeros((B, 160, H, d), dtype=q.dtype, device="cuda"), torch.zeros((B, 160, H, d), dtype=q.dtype, device="cuda")] for _ in range(2)]
    ws = [fa.new_q8_workspace(made[0][0], n) for _ in range(2)]

    def run(i, stream=None):
        lay, cache = made[i]
        fa.fa_q8_append(lay, cache, K, V, count, stream=stream)
        fa.fa_q8_attention(lay, cache, q, outs[i][0], ws[i], stream=stream)
        fa.fa_q8_read(lay, cache, outs[i][1], outs[i][2], stream=stream)

    run(1)                                                             # (the first calls set the kernels' attributes)
    fa.fa_q8_reset(*made[1])
    torch.cuda.synchronize()
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        run(0, side)
    for i in range(7):                                                 # the last one is refused for row 0: 168 tokens
        K.copy_(rand(K.shape, "bf16", 10 + i))
        q.copy_(rand(q.shape, "bf16", 30 + i))
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            graph.replay()
        torch.cuda.synchronize()
        run(1)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(*outs)), i
        assert made[0][1].state[:, 0].tolist() == made[1][1].state[:, 0].tolist() == [min(24 * (i + 1), 144), 19 * (i + 1)]
    assert [fa.fa_q8_poll_status(c) for _, c in made] == [fa.FA_ERR_CAPACITY] * 2

"""The dense cache in 8 bits (fa_q8_*) against its 64-bit statement in tests/q8_reference.py."""
import math

import numpy as np
import pytest
import torch

from paper_2506_11886_b200 import fa, synth
from tests import q8_reference as ref

pytestmark = pytest.mark.gpu
FMT = {"int8": fa.FA_Q8_INT8, "e4m3": fa.FA_Q8_E4M3}
DT = {"bf16": (torch.bfloat16, fa.FA_BF16), "f32": (torch.float32, fa.FA_F32)}


def make(B=1, Hq=8, H=2, d=128, block=32, nb=8, fmt="int8", dtype="bf16", scale=None, seed=0, shuffle=True, extra=2):
    lay = fa.Q8Layout(batch=B, n_q_heads=Hq, n_kv_heads=H, head_dim=d, block=block, max_blocks=nb, n_pages=B * nb + extra, format=FMT[fmt],
                      kv_dtype=DT[dtype][1], softmax_scale=d ** -0.5 if scale is None else scale)
    cache = fa.Q8Cache(lay)
    if shuffle:
        g = torch.Generator().manual_seed(seed)
        cache.block_table.copy_(torch.randperm(lay.n_pages, generator=g)[:B * nb].reshape(B, nb).to(torch.int32))
    return lay, cache


def rand(shape, dtype, seed, spread=0.5):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(shape, generator=g) * torch.exp(spread * torch.randn(shape[-1], generator=g))
    return x.to(DT[dtype][0]).cuda()


def check_cache(lay, cache, rows, fmt):
    """Every page that the rows hold, its scale, the tails and the lengths, bit for bit."""
    torch.cuda.synchronize()
    assert fa.fa_q8_poll_status(cache) == fa.FA_OK
    state = cache.state.cpu()
    assert state[:, 0].tolist() == [k.shape[0] for k in rows.k] and (state[:, 1:] == 0).all() and (cache.status == 0).all()
    table = cache.block_table.cpu()
    for side in ("k", "v"):
        pages, scales, tail = (getattr(cache, f"{side}_{n}").cpu() for n in ("pages", "scale", "tail"))
        for b, x in enumerate(getattr(rows, side)):
            n = x.shape[0]
            for h in range(lay.n_kv_heads):
                for i in range(n // lay.block):
                    blk = rows.block_of(side, b, h, i)
                    want = ref.scale32(blk, fmt)
                    got = float(scales[table[b, i], h])
                    assert got == want or (math.isnan(got) and math.isnan(want)), (side, b, h, i, got, want)
                    codes = pages[table[b, i], h].to(torch.float64)
                    if not math.isnan(want):
                        assert torch.equal(codes, ref.codes(blk, fmt)), (side, b, h, i)
                r = n % lay.block
                if r:
                    assert torch.equal(tail[b, h, :r].view(torch.uint8), x[n - r:, h].contiguous().view(torch.uint8)), (side, b, h)
                    if torch.isfinite(x[n - r:, h].float()).all():
                        assert float(cache.tail_amax[b, h, 0 if side == "k" else 1]) == float(x[n - r:, h].float().abs().max())


# ---- writing ----------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d,block", [(64, 16), (128, 32), (128, 128), (256, 64), (256, 128)])
def test_write_rounds_complete_blocks_and_keeps_the_rest(fmt, dtype, d, block):
    n = 3 * block + 5
    lens = [n, 0, block, 2 * block - 1, 1]
    lay, cache = make(B=5, H=2, d=d, block=block, nb=4, fmt=fmt, dtype=dtype)
    K, V = rand((5, n, 2, d), dtype, 1), rand((5, n, 2, d), dtype, 2)
    fa.fa_q8_write(lay, cache, K, V, torch.tensor(lens, dtype=torch.int32, device="cuda"))
    rows = ref.Rows(5, 2, d, block, fmt, DT[dtype][0])
    for b, m in enumerate(lens):
        rows.push(b, K[b, :m], V[b, :m])
    check_cache(lay, cache, rows, fmt)


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_half_way_values_go_to_even(fmt, dtype):
    """Blocks whose quotients lie on, and one unit beside, the borders between two 8-bit numbers, for many largest magnitudes."""
    d, block, nb = 64, 16, 64
    lay, cache = make(d=d, block=block, nb=nb, H=1, Hq=1, fmt=fmt, dtype=dtype)
    bits = 8 if dtype == "bf16" else 24
    blocks = []
    g = torch.Generator().manual_seed(5)
    for i in range(nb):
        top = ref.TOP[fmt]
        # magnitudes that make ties: multiples of the top's odd factor, powers of two, others
        amax = float([127, 254, 224, 192, 1.0, 3.0, 7 * 2.0 ** -20, 160][i % 8]) * (1 + (i // 8) * 2.0 ** -7)
        j = torch.randint(-127 if fmt == "int8" else -224, 127 if fmt == "int8" else 224, (block * d,), generator=g).double() + 0.5
        x = (j / top * amax).to(DT[dtype][0]).double()
        x[::3] = torch.nextafter(x[::3].float(), torch.tensor(float("inf"))).to(DT[dtype][0]).double()
        x = x.clamp(-amax, amax)
        x[7] = amax
        blocks.append(x.reshape(block, 1, d))
    K = torch.cat(blocks).to(DT[dtype][0])[None].cuda()
    fa.fa_q8_write(lay, cache, K, -K)
    rows = ref.Rows(1, 1, d, block, fmt, DT[dtype][0])
    rows.push(0, K[0], -K[0])
    check_cache(lay, cache, rows, fmt)


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_blocks_of_any_magnitude(fmt, dtype):
    """Zeros, the smallest and the largest numbers, one value, infinities and NaN: a block of its own each."""
    d, block, H = 64, 16, 1
    fin = torch.finfo(DT[dtype][0])
    tiny = fin.tiny * fin.eps
    g = torch.Generator().manual_seed(3)
    base = torch.randn((block, d), generator=g)
    blocks = [base * 0, base * 1e-38, torch.full_like(base, tiny), base * 1e-20, base * 1e20, (base / base.abs().max()) * fin.max,
              torch.where(torch.arange(d) == 5, 1e-30, 0.0).expand(block, d), torch.where(torch.arange(d) == 5, fin.max, base * tiny),
              torch.where(torch.arange(d) == 5, math.inf, base), torch.where(torch.arange(d) == 5, -math.inf, base), torch.where(torch.arange(d) == 5, math.nan, base)]
    lay, cache = make(d=d, block=block, nb=len(blocks), H=H, Hq=1, fmt=fmt, dtype=dtype)
    K = torch.cat(blocks).to(DT[dtype][0]).reshape(1, -1, 1, d).cuda()
    assert torch.isfinite(K[0, :8 * block].float()).all()
    fa.fa_q8_write(lay, cache, K, K.flip(3))
    rows = ref.Rows(1, 1, d, block, fmt, DT[dtype][0])
    rows.push(0, K[0], K[0].flip(2))
    check_cache(lay, cache, rows, fmt)
    k, v = torch.zeros_like(K), torch.zeros_like(K)
    fa.fa_q8_read(lay, cache, k, v)
    assert torch.isnan(k[0, 8 * block:].float()).all() and torch.isfinite(k[0, :8 * block].float()).all()


@pytest.mark.parametrize("block", [16, 128])
def test_the_cache_does_not_depend_on_the_calls(block):
    """One write, appends of chunks of all sorts (ragged, empty, past several blocks), steps: the same pages, tails, lengths."""
    B, H, d, fmt, dtype = 3, 2, 128, "e4m3", "bf16"
    total = 4 * block + 3
    K, V = rand((B, total, H, d), dtype, 1), rand((B, total, H, d), dtype, 2)
    rows = ref.Rows(B, H, d, block, fmt, torch.bfloat16)
    lay, cache = make(B=B, Hq=4, H=H, d=d, block=block, nb=5, fmt=fmt, dtype=dtype)
    fa.fa_q8_reset(lay, cache)
    have = [0] * B
    rng = np.random.default_rng(0)
    sizes = [1, block - 1, 0, block, 2, block + 1, 5, block // 2, 2 * block]
    while min(have) < total:
        n = int(sizes[rng.integers(len(sizes))])
        want = [int(min(total - have[b], rng.integers(0, n + 1) if rng.random() < 0.5 else n)) for b in range(B)]
        k, v = torch.full((B, n, H, d), float("nan"), dtype=torch.bfloat16, device="cuda"), torch.full((B, n, H, d), float("nan"), dtype=torch.bfloat16, device="cuda")
        for b, m in enumerate(want):
            k[b, :m], v[b, :m] = K[b, have[b]:have[b] + m], V[b, have[b]:have[b] + m]
            rows.push(b, k[b, :m], v[b, :m])
            have[b] += m
        fa.fa_q8_append(lay, cache, k, v, torch.tensor(want, dtype=torch.int32, device="cuda"))
        check_cache(lay, cache, rows, fmt)
    lay2, once = make(B=B, Hq=4, H=H, d=d, block=block, nb=5, fmt=fmt, dtype=dtype)
    fa.fa_q8_write(lay2, once, K, V)
    for side in ("k", "v"):
        for b in range(B):
            at = once.block_table[b, :total // block].long()
            assert torch.equal(getattr(once, side + "_pages").view(torch.uint8)[at], getattr(cache, side + "_pages").view(torch.uint8)[at])
            assert torch.equal(getattr(once, side + "_scale")[at], getattr(cache, side + "_scale")[at])


def test_tokens_of_a_fused_projection():
    """K and V as slices of one [B][n][(Hq + 2 H) d] projection: strides that are none of the layout's."""
    B, n, Hq, H, d, block = 2, 70, 6, 3, 64, 32
    lay, cache = make(B=B, Hq=Hq, H=H, d=d, block=block, nb=3)
    qkv = rand((B, n, Hq + 2 * H, d), "bf16", 4)
    K, V = qkv[:, :, Hq:Hq + H], qkv[:, :, Hq + H:]
    fa.fa_q8_write(lay, cache, K, V)
    rows = ref.Rows(B, H, d, block, "int8", torch.bfloat16)
    for b in range(B):
        rows.push(b, K[b], V[b])
    check_cache(lay, cache, rows, "int8")


def test_rows_that_do_not_fit_and_pages_that_are_not_there():
    B, H, d, block, nb = 4, 2, 64, 16, 3
    lay, cache = make(B=B, H=H, d=d, block=block, nb=nb)
    K, V = rand((B, 40, H, d), "bf16", 1), rand((B, 40, H, d), "bf16", 2)
    n0 = [40, 9, 20, 30]
    fa.fa_q8_write(lay, cache, K, V, torch.tensor(n0, dtype=torch.int32, device="cuda"))
    rows = ref.Rows(B, H, d, block, "int8", torch.bfloat16)
    for b in range(B):
        rows.push(b, K[b, :n0[b]], V[b, :n0[b]])
    check_cache(lay, cache, rows, "int8")
    # row 0 has room for 8 more only; row 1 gets its 9; row 2 would complete a block without a page; row 3 has one that needs none
    good = cache.block_table.clone()
    cache.block_table[2, 1], cache.block_table[3, 2] = lay.n_pages, -1
    k, v = rand((B, 13, H, d), "bf16", 3), rand((B, 13, H, d), "bf16", 4)
    fa.fa_q8_append(lay, cache, k, v, torch.tensor([9, 9, 13, 2], dtype=torch.int32, device="cuda"))
    assert fa.fa_q8_poll_status(cache) in (fa.FA_ERR_CAPACITY, fa.FA_ERR_INDEX)
    cache.block_table.copy_(good)
    rows.push(1, k[1, :9], v[1, :9])
    rows.push(3, k[3, :2], v[3, :2])
    check_cache(lay, cache, rows, "int8")
    fa.fa_q8_append(lay, cache, k, v, torch.tensor([8, 99, -5, 13], dtype=torch.int32, device="cuda"))      # counts are clamped to 0 .. n
    for b, m in ((0, 8), (1, 13), (3, 13)):
        rows.push(b, k[b, :m], v[b, :m])
    check_cache(lay, cache, rows, "int8")
    # a write without a page leaves the row empty, one that is too long leaves it alone
    cache.block_table[1, 0] = -7
    fa.fa_q8_write(lay, cache, k, v)
    assert fa.fa_q8_poll_status(cache) == fa.FA_OK                                                    # 13 tokens complete no block
    fa.fa_q8_write(lay, cache, K, V, torch.tensor([40, 40, 5, 40], dtype=torch.int32, device="cuda"))
    assert fa.fa_q8_poll_status(cache) == fa.FA_ERR_INDEX
    assert cache.state[:, 0].tolist() == [40, 0, 5, 40]
    cache.state[2, 0] = lay.max_blocks * block + 1                                                    # not a length
    fa.fa_q8_append(lay, cache, k, v)
    assert fa.fa_q8_poll_status(cache) == fa.FA_ERR_CAPACITY


# ---- reading ----------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d,block,t0,n", [(64, 16, 0, 100), (128, 64, 37, 150), (256, 32, 95, 1), (128, 128, 130, 60), (64, 32, 150, 100)])
def test_read_gives_what_the_cache_stands_for(fmt, dtype, d, block, t0, n):
    """A value is code * scale with one rounding, and one to the dtype: half a step of fp32 for the scale, the product, then
    half a step of the dtype.  Tokens that a row does not hold, and what lies around the output, stay as they were."""
    B, H = 3, 2
    lens = [187, 0, 96]
    lay, cache = make(B=B, H=H, d=d, block=block, nb=-(-187 // block), fmt=fmt, dtype=dtype)
    K, V = rand((B, 187, H, d), dtype, 1), rand((B, 187, H, d), dtype, 2)
    fa.fa_q8_write(lay, cache, K, V, torch.tensor(lens, dtype=torch.int32, device="cuda"))
    rows = ref.Rows(B, H, d, block, fmt, DT[dtype][0])
    for b in range(B):
        rows.push(b, K[b, :lens[b]], V[b, :lens[b]])
    big = torch.full((2, B, n + 2, H + 1, d), -77.0, dtype=DT[dtype][0], device="cuda")
    fa.fa_q8_read(lay, cache, big[0, :, 1:n + 1, :H], big[1, :, 1:n + 1, :H], t0)
    assert fa.fa_q8_poll_status(cache) == fa.FA_OK
    got = big.cpu().double()
    assert (got[:, :, 0] == -77).all() and (got[:, :, -1] == -77).all() and (got[:, :, :, H] == -77).all()
    rel = 2.0 ** -24 * 2 + torch.finfo(DT[dtype][0]).eps / 2
    for i, side in enumerate("kv"):
        for b in range(B):
            there = max(0, min(n, lens[b] - t0))
            assert (got[i, b, 1 + there:] == -77).all()
            for h in range(H):
                want = rows.held(side, b, h)[t0:t0 + there]
                assert ((got[i, b, 1:1 + there, h] - want).abs() <= rel * want.abs()).all()


# ---- attention --------------------------------------------------------------------------------------------------------
def attend_and_check(lay, cache, rows, q, dtype, ws=None, view=None):
    n_q = q.shape[1]
    out = torch.full(q.shape, float("nan"), dtype=q.dtype, device="cuda")
    ws = fa.new_q8_workspace(lay, n_q) if ws is None else ws
    fa.fa_q8_attention(lay, cache, q if view is None else view, out, ws)
    torch.cuda.synchronize()
    assert fa.fa_q8_poll_status(cache) == fa.FA_OK
    assert (ws[:4096] == 0).all()
    got, G = out.cpu().double(), lay.n_q_heads // lay.n_kv_heads
    worst = 0.0
    for b in range(lay.batch):
        for h in range(lay.n_kv_heads):
            k, v = rows.held("k", b, h), rows.held("v", b, h)
            want, tol = ref.attention(k, v, q[b, :, h * G:(h + 1) * G].cpu().double(), n_q, lay.softmax_scale, DT[dtype][0])
            err = (got[b, :, h * G:(h + 1) * G] - want).abs()
            assert (err <= tol).all(), (b, h, float((err / tol).max()), float(err.max()))
            worst = max(worst, float((err / tol).max()))
    return out, worst


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("Hq,H,d,block,n_q", [
    (8, 2, 128, 64, 1), (2, 2, 64, 16, 1), (16, 1, 128, 32, 1), (6, 2, 256, 128, 1), (3, 1, 64, 128, 1), (32, 2, 256, 16, 1),
    (8, 2, 128, 32, 5), (4, 4, 64, 64, 7), (12, 4, 128, 16, 11), (2, 1, 256, 64, 33)])
def test_attention_matches_its_definition(fmt, dtype, Hq, H, d, block, n_q):
    """Rows of every sort of length: none, one token, around a unit of 16, around a block, several parts, all of the capacity."""
    lens = [0, 1, 15, 16, 17, block - 1, block, block + 1, 3 * block + 5, 700, 1024]
    nb = 1024 // block
    B = len(lens)
    lay, cache = make(B=B, Hq=Hq, H=H, d=d, block=block, nb=nb, fmt=fmt, dtype=dtype)
    K, V = rand((B, 1024, H, d), dtype, 1), rand((B, 1024, H, d), dtype, 2)
    fa.fa_q8_write(lay, cache, K, V, torch.tensor(lens, dtype=torch.int32, device="cuda"))
    rows = ref.Rows(B, H, d, block, fmt, DT[dtype][0])
    for b in range(B):
        rows.push(b, K[b, :lens[b]], V[b, :lens[b]])
    q = rand((B, n_q, Hq, d), dtype, 3)
    out, _ = attend_and_check(lay, cache, rows, q, dtype)
    assert (out[0] == 0).all()
    # the same queries as a slice of a wider projection, bit for bit
    wide = torch.full((B, n_q, Hq + 3, d), float("nan"), dtype=q.dtype, device="cuda")
    wide[:, :, 1:1 + Hq] = q
    again, _ = attend_and_check(lay, cache, rows, q, dtype, view=wide[:, :, 1:1 + Hq])
    assert torch.equal(out, again)


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
@pytest.mark.parametrize("Hq,H,d,block,n_q", [(8, 2, 128, 64, 100), (4, 1, 64, 16, 16), (3, 3, 64, 128, 257), (12, 4, 128, 16, 200), (16, 1, 128, 128, 33), (4, 2, 128, 32, 640)])
def test_chunks_of_queries_match_their_definition(fmt, Hq, H, d, block, n_q):
    """Rows shorter than the chunk, empty, around a tile of 128 tokens and a block, cut into several parts; tiles of queries that are not full."""
    lens = [0, 1, 17, 127, 128, 129, n_q, n_q + 1, 5 * block + 3, 1000]
    B, most = len(lens), 1024
    lay, cache = make(B=B, Hq=Hq, H=H, d=d, block=block, nb=most // block, fmt=fmt)
    K, V = rand((B, most, H, d), "bf16", 1), rand((B, most, H, d), "bf16", 2)
    fa.fa_q8_write(lay, cache, K, V, torch.tensor(lens, dtype=torch.int32, device="cuda"))
    rows = ref.Rows(B, H, d, block, fmt, torch.bfloat16)
    for b in range(B):
        rows.push(b, K[b, :lens[b]], V[b, :lens[b]])
    q = rand((B, n_q, Hq, d), "bf16", 3)
    out, _ = attend_and_check(lay, cache, rows, q, "bf16")
    assert (out[0] == 0).all()
    wide = torch.full((B, n_q, Hq + 3, d), float("nan"), dtype=q.dtype, device="cuda")
    wide[:, :, 1:1 + Hq] = q
    again, _ = attend_and_check(lay, cache, rows, q, "bf16", view=wide[:, :, 1:1 + Hq])
    assert torch.equal(out, again)


def test_a_long_row_and_one_tile_of_queries():
    """One tile of queries over 30 000 tokens, cut into as many parts as there are SMs; blocks of very different scales."""
    Hq, H, d, block, n = 4, 1, 128, 64, 30000
    lay, cache = make(Hq=Hq, H=H, d=d, block=block, nb=470)
    K, V = rand((1, n, H, d), "bf16", 1), rand((1, n, H, d), "bf16", 2)
    V = (V.float() * 10.0 ** (torch.arange(n, device="cuda") // 700 % 13 - 6)[None, :, None, None]).bfloat16()
    fa.fa_q8_write(lay, cache, K, V)
    rows = ref.Rows(1, H, d, block, "int8", torch.bfloat16)
    rows.push(0, K[0], V[0])
    attend_and_check(lay, cache, rows, rand((1, 40, Hq, d), "bf16", 3), "bf16")


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
def test_long_rows_and_many_parts(fmt):
    """A row of 20 001 tokens in many parts beside a short one; nearly equal and very different scores."""
    B, Hq, H, d, block = 2, 8, 2, 128, 64
    for spread, scale in ((0.0, 1e-4), (0.5, 1.0)):
        lay, cache = make(B=B, Hq=Hq, H=H, d=d, block=block, nb=320, fmt=fmt, scale=scale)
        K, V = rand((B, 20001, H, d), "bf16", 1, spread), rand((B, 20001, H, d), "bf16", 2)
        lens = [20001, 130]
        fa.fa_q8_write(lay, cache, K, V, torch.tensor(lens, dtype=torch.int32, device="cuda"))
        rows = ref.Rows(B, H, d, block, fmt, torch.bfloat16)
        for b in range(B):
            rows.push(b, K[b, :lens[b]], V[b, :lens[b]])
        attend_and_check(lay, cache, rows, rand((B, 1, Hq, d), "bf16", 3), "bf16")


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
def test_fp32_sums_over_long_rows_are_rounded_not_cut_off(fmt):
    """q = 0, so every weight is 1 and a column's output the mean of its V, all of one sign: errors of one direction add up.
    A warp sums about 700 units of 16 tokens.  Counted: weights in two halves 2^-22, the sums inside the MMAs of a unit 4 x 2^-23,
    the join and the division 25 x 2^-24, and 700 additions rounded by at most 2^-24 of a sum that grows to the last one's
    size, of either sign: a deviation of sqrt(700 / 3) / sqrt(3) x 2^-24 and six of those.  (Cut off instead: 700 x 2^-24.)"""
    B, H, d, block, nb = 40, 4, 64, 128, 640
    n = nb * block
    one, src = make(B=1, Hq=H, H=H, d=d, block=block, nb=nb, fmt=fmt, dtype="f32")
    V = rand((1, n, H, d), "f32", 1).abs() + 0.25
    fa.fa_q8_write(one, src, V.flip(1), V)
    lay = fa.Q8Layout(batch=B, n_q_heads=H, n_kv_heads=H, head_dim=d, block=block, max_blocks=nb, n_pages=one.n_pages, format=FMT[fmt],
                      kv_dtype=fa.FA_F32, softmax_scale=0.125)
    cache = fa.Q8Cache(lay)
    for name in ("k_pages", "v_pages", "k_scale", "v_scale"):
        getattr(cache, name).copy_(getattr(src, name))
    cache.block_table.copy_(src.block_table.expand(B, nb))
    cache.state[:, 0] = n
    q = torch.zeros((B, 1, H, d), device="cuda")
    out = torch.full_like(q, math.nan)
    fa.fa_q8_attention(lay, cache, q, out, fa.new_q8_workspace(lay))
    assert fa.fa_q8_poll_status(cache) == fa.FA_OK
    page = src.block_table[0].long()
    want = torch.zeros((H, d), dtype=torch.float64, device="cuda")
    for i in range(nb):
        want += src.v_pages[page[i]].double().sum(1) * src.v_scale[page[i]].double()[:, None]
    want /= n
    err = ((out.double().reshape(B, H, d) - want) / want).abs().max()
    assert float(err) <= 2.0 ** -22 + 4 * 2.0 ** -23 + 25 * 2.0 ** -24 + 6 * math.sqrt(700 / 9) * 2.0 ** -24


@pytest.mark.parametrize("fmt,d", [("int8", 128), ("e4m3", 64)])
def test_a_chunk_at_the_end_of_a_million_tokens(fmt, d):
    """q = 0: a column's output is the mean of its V, all of one sign.  A tile is summed by one or two CTAs over 8192 blocks of 128 tokens.
    Counted: the output's half step, the weights' (halves, 2^-11), cut-offs of 2^-13 in runs of 256 blocks and 2^-13 for all that is rounded to 2^-24."""
    B, H, G, block, held, nb, n_q = 2, 2, 8, 128, 512, 8192, 1024
    n = nb * block
    one, src = make(B=1, Hq=H, H=H, d=d, block=block, nb=held, fmt=fmt, extra=0)
    V = (rand((1, held * block, H, d), "f32", 1, 0.0).abs() + 0.25).bfloat16()
    fa.fa_q8_write(one, src, V, V)
    lay = fa.Q8Layout(batch=B, n_q_heads=G * H, n_kv_heads=H, head_dim=d, block=block, max_blocks=nb, n_pages=held, format=FMT[fmt],
                      kv_dtype=fa.FA_BF16, softmax_scale=0.125)
    cache = fa.Q8Cache(lay)
    for name in ("k_pages", "v_pages", "k_scale", "v_scale"):
        getattr(cache, name).copy_(getattr(src, name))
    table = torch.randint(0, held, (nb,), generator=torch.Generator().manual_seed(1))
    cache.block_table.copy_(table.to(torch.int32).expand(B, nb))
    cache.state[:, 0] = n
    q = torch.zeros((B, n_q, G * H, d), dtype=torch.bfloat16, device="cuda")
    out = torch.full_like(q, math.nan)
    fa.fa_q8_attention(lay, cache, q, out, fa.new_q8_workspace(lay, n_q))
    assert fa.fa_q8_poll_status(cache) == fa.FA_OK
    block_sums = src.v_pages.double().sum(2) * src.v_scale.double()[:, :, None]
    # all queries see the blocks in front of the last eight; the last one all of them
    want = (block_sums * torch.bincount(table, minlength=held).double().cuda()[:, None, None]).sum(0) / n
    err = ((out[:, -1].double().reshape(B, H, G, d) - want[None, :, None]) / want[None, :, None]).abs().max()
    assert float(err) <= 2.0 ** -8 + 2.0 ** -11 + 2.0 ** -13 + 2.0 ** -13
    # ... the first one the tokens up to its own
    seen = n - n_q + 1
    want = ((want * n) - sum(block_sums[table[i]] for i in range(nb - 8, nb)) + src.v_pages[table[nb - 8], :, 0].double() * src.v_scale[table[nb - 8]].double()[:, None]) / seen
    err = ((out[:, 0].double().reshape(B, H, G, d) - want[None, :, None]) / want[None, :, None]).abs().max()
    assert float(err) <= 2.0 ** -8 + 2.0 ** -11 + 2.0 ** -13 + 2.0 ** -13


@pytest.mark.parametrize("scores", [3.0, 40.0])
def test_runs_of_blocks_with_maxima_that_grow(scores):
    """The sums of 256 blocks are put away while the maxima of the scores and of the values still grow, in tiles of one CTA and in cut ones."""
    B, Hq, H, d, block, n, n_q = 170, 8, 1, 64, 64, 80000, 9
    one, src = make(Hq=Hq, H=H, d=d, block=block, nb=1250, scale=1.0)
    K, V = rand((1, n, H, d), "bf16", 1, 0.0), rand((1, n, H, d), "bf16", 2, 0.0)
    ramp = torch.linspace(0.05, 1.0, n, device="cuda")[None, :, None, None]
    K = (K.float() * ramp * scores / 24).bfloat16()
    V = (V.float() * 2.0 ** (torch.arange(n, device="cuda") // 9000 - 4)[None, :, None, None]).bfloat16()
    fa.fa_q8_write(one, src, K, V)
    lay = fa.Q8Layout(batch=B, n_q_heads=Hq, n_kv_heads=H, head_dim=d, block=block, max_blocks=1250, n_pages=one.n_pages, format=fa.FA_Q8_INT8,
                      kv_dtype=fa.FA_BF16, softmax_scale=1.0)
    cache = fa.Q8Cache(lay)
    for name in ("k_pages", "v_pages", "k_scale", "v_scale"):
        getattr(cache, name).copy_(getattr(src, name))
    cache.block_table.copy_(src.block_table.expand(B, 1250))
    cache.state[:, 0] = n
    rows = ref.Rows(1, H, d, block, "int8", torch.bfloat16)
    rows.push(0, K[0], V[0])
    k, v = rows.held("k", 0, 0), rows.held("v", 0, 0)
    q = rand((B, n_q, Hq, d), "bf16", 3, 0.0)
    out = torch.full_like(q, math.nan)
    fa.fa_q8_attention(lay, cache, q, out, fa.new_q8_workspace(lay, n_q))
    assert fa.fa_q8_poll_status(cache) == fa.FA_OK
    assert torch.isfinite(out.float()).all()
    for b in (0, 1, 60, 85, 118, 168, 169):
        want, tol = ref.attention(k, v, q[b].cpu().double(), n_q, 1.0, torch.bfloat16)
        err = (out[b].cpu().double() - want).abs()
        assert (err <= tol).all(), (b, float((err / tol).max()))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_blocks_of_very_different_scale(dtype):
    """V blocks (and a tail) from 1e-30 to 1e30, K blocks from 1e-6 on: a weight's share in the result goes by p times its block's scale."""
    Hq, H, d, block, n = 4, 1, 64, 16, 16 * 12 + 9
    lay, cache = make(Hq=Hq, H=H, d=d, block=block, nb=13, dtype=dtype)
    for order in (1, -1):
        f = 10.0 ** (order * torch.linspace(-30, 30, 13))
        fk = 10.0 ** torch.linspace(-6, 0, 13)
        K, V = rand((1, n, H, d), dtype, 1).float().cpu(), rand((1, n, H, d), dtype, 2).float().cpu()
        K *= fk.repeat_interleave(block)[None, :n, None, None]
        V *= f.repeat_interleave(block)[None, :n, None, None]
        K, V = K.to(DT[dtype][0]).cuda(), V.to(DT[dtype][0]).cuda()
        fa.fa_q8_write(lay, cache, K, V)
        rows = ref.Rows(1, H, d, block, "int8", DT[dtype][0])
        rows.push(0, K[0], V[0])
        attend_and_check(lay, cache, rows, rand((1, 1, Hq, d), dtype, 3), dtype)
    # the large scores lie on blocks of small V
    K = torch.where(torch.arange(n)[None, :, None, None] < 64, 3.0, -3.0).expand(1, n, H, d).to(DT[dtype][0]).contiguous().cuda()
    V = (rand((1, n, H, d), dtype, 2).cpu().float() * torch.where(torch.arange(n)[None, :, None, None] < 64, 1e-12, 1.0)).to(DT[dtype][0]).cuda()
    fa.fa_q8_write(lay, cache, K, V)
    rows = ref.Rows(1, H, d, block, "int8", DT[dtype][0])
    rows.push(0, K[0], V[0])
    attend_and_check(lay, cache, rows, torch.full((1, 1, Hq, d), 0.5, dtype=DT[dtype][0], device="cuda"), dtype)


def test_what_is_behind_the_row_has_no_effect():
    """NaN in the tail behind the row's last token, in pages of later blocks and of nobody, in the scales: bit for bit the same."""
    B, Hq, H, d, block, fmt = 2, 8, 2, 128, 32, "e4m3"
    lay, cache = make(B=B, Hq=Hq, H=H, d=d, block=block, nb=6, fmt=fmt)
    K, V = rand((B, 100, H, d), "bf16", 1), rand((B, 100, H, d), "bf16", 2)
    lens = torch.tensor([100, 70], dtype=torch.int32, device="cuda")
    fa.fa_q8_write(lay, cache, K, V, lens)
    q, ws = rand((B, 4, Hq, d), "bf16", 3), fa.new_q8_workspace(lay, 4)
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
    # a later block that is not finite is NaN for the queries that see it, and for no other
    K[0, 97], V[0, 97] = float("inf"), float("nan")
    good = make(B=B, Hq=Hq, H=H, d=d, block=block, nb=6, fmt=fmt)[1]
    fa.fa_q8_write(lay, good, K, V, lens)
    fa.fa_q8_attention(lay, good, q, dirty, ws)
    assert torch.equal(out[1], dirty[1]) and torch.isnan(dirty[0, 1:].float()).all()


def test_pages_out_of_range_are_left_out_and_reported():
    Hq, H, d, block = 4, 1, 64, 16
    lay, cache = make(Hq=Hq, H=H, d=d, block=block, nb=8)
    K, V = rand((1, 100, H, d), "bf16", 1), rand((1, 100, H, d), "bf16", 2)
    fa.fa_q8_write(lay, cache, K, V)
    cache.block_table[0, 1], cache.block_table[0, 4] = -1, lay.n_pages
    q = rand((1, 1, Hq, d), "bf16", 3)
    out, ws = torch.empty_like(q), fa.new_q8_workspace(lay)
    fa.fa_q8_attention(lay, cache, q, out, ws)
    assert fa.fa_q8_poll_status(cache) == fa.FA_ERR_INDEX
    rows = ref.Rows(1, H, d, block, "int8", torch.bfloat16)
    rows.push(0, K[0], V[0])
    keep = [t for t in range(100) if t // block not in (1, 4)]
    want, tol = ref.attention(rows.held("k", 0, 0)[keep], rows.held("v", 0, 0)[keep], q[0].cpu().double(), 1, lay.softmax_scale, torch.bfloat16)
    assert ((out[0].cpu().double() - want).abs() <= tol).all()
    k = torch.full_like(K, -5.0)
    v = k.clone()
    fa.fa_q8_read(lay, cache, k, v)
    assert fa.fa_q8_poll_status(cache) == fa.FA_ERR_INDEX
    gone = torch.tensor([t // block in (1, 4) for t in range(100)])
    assert (k[0, gone] == -5).all() and (k[0, ~gone] != -5).any(-1).all()


def test_rows_may_share_pages_and_pages_may_lie_past_32_bits():
    """A common prompt of two blocks, read through the same pages by two rows; the pages are the last of 4.5 GB."""
    Hq, H, d, block = 8, 8, 128, 128
    n_pages = 36_000
    lay = fa.Q8Layout(batch=2, n_q_heads=Hq, n_kv_heads=H, head_dim=d, block=block, max_blocks=4, n_pages=n_pages, softmax_scale=0.1)
    pages = [torch.empty((n_pages, H, block, d), dtype=torch.int8, device="cuda") for _ in range(2)]
    assert pages[0].numel() > 1 << 32
    cache = fa.Q8Cache(lay, buffers=dict(k_pages=pages[0], v_pages=pages[1]))
    cache.block_table.copy_(torch.tensor([[n_pages - 1, n_pages - 3, 5, 6], [n_pages - 1, n_pages - 3, n_pages - 2, 7]], dtype=torch.int32))
    K, V = rand((2, 400, H, d), "bf16", 1), rand((2, 400, H, d), "bf16", 2)
    K[1, :256], V[1, :256] = K[0, :256], V[0, :256]
    lens = [300, 400]
    fa.fa_q8_write(lay, cache, K, V, torch.tensor(lens, dtype=torch.int32, device="cuda"))      # (both write the same bytes to the shared pages)
    rows = ref.Rows(2, H, d, block, "int8", torch.bfloat16)
    for b in range(2):
        rows.push(b, K[b, :lens[b]], V[b, :lens[b]])
    torch.cuda.synchronize()
    attend_and_check(lay, cache, rows, rand((2, 1, Hq, d), "bf16", 3), "bf16")
    k, v = torch.zeros_like(K), torch.zeros_like(K)
    fa.fa_q8_read(lay, cache, k, v)
    assert torch.equal(k[0, :256], k[1, :256]) and (k[1, 256:384] != 0).any()


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
@pytest.mark.parametrize("n_q", [1, 40])
def test_pages_of_an_engine(fmt, n_q):
    """Pages, scales and lengths that did not come from fa_q8_write: any byte (int8 -128 among them; no e4m3 NaN), scales of zero; more than 32 rows."""
    B, Hq, H, d, block, nb = 40, 4, 2, 128, 32, 6
    lay, cache = make(B=B, Hq=Hq, H=H, d=d, block=block, nb=nb, fmt=fmt)
    g = torch.Generator().manual_seed(9)
    for side in ("k", "v"):
        raw = torch.randint(0, 256, getattr(cache, side + "_pages").shape, generator=g, dtype=torch.uint8)
        if fmt == "e4m3":
            raw[(raw & 0x7f) == 0x7f] = 0x70
        getattr(cache, side + "_pages").view(torch.uint8).copy_(raw)
        scale = 0.02 * torch.rand(getattr(cache, side + "_scale").shape, generator=g)
        scale[::7] = 0
        getattr(cache, side + "_scale").copy_(scale)
    lens = [(b * 37) % (nb * block) // block * block for b in range(B)]
    cache.state[:, 0] = torch.tensor(lens, dtype=torch.int32)
    q = rand((B, n_q, Hq, d), "bf16", 3)
    out, ws = torch.full_like(q, float("nan")), fa.new_q8_workspace(lay, n_q)
    fa.fa_q8_attention(lay, cache, q, out, ws)
    assert fa.fa_q8_poll_status(cache) == fa.FA_OK
    table, got = cache.block_table.cpu().long(), out.cpu().double()
    for b in range(B):
        for h in range(H):
            kv = [getattr(cache, s + "_pages")[:, h].cpu()[table[b, :lens[b] // block]].double() * getattr(cache, s + "_scale")[:, h].cpu()[table[b, :lens[b] // block]].double()[:, None, None]
                  for s in ("k", "v")]
            k, v = (x.reshape(lens[b], d) for x in kv)
            want, tol = ref.attention(k, v, q[b, :, 2 * h:2 * h + 2].cpu().double(), n_q, lay.softmax_scale, torch.bfloat16)
            assert ((got[b, :, 2 * h:2 * h + 2] - want).abs() <= tol).all(), (b, h)


def test_a_length_that_is_none_is_refused_row_by_row():
    lay, cache = make(B=3, H=2, d=64, block=16, nb=2)
    K = rand((3, 32, 2, 64), "bf16", 1)
    fa.fa_q8_write(lay, cache, K, K)
    cache.state[0, 0], cache.state[2, 0] = 33, -1
    q = rand((3, 1, 8, 64), "bf16", 2)
    out, ws = torch.full_like(q, float("nan")), fa.new_q8_workspace(lay)
    fa.fa_q8_attention(lay, cache, q, out, ws)
    assert fa.fa_q8_poll_status(cache) == fa.FA_ERR_CAPACITY
    assert (out[0] == 0).all() and (out[2] == 0).all() and torch.isfinite(out[1].float()).all() and (out[1] != 0).any()
    k = torch.full_like(K, -3.0)
    fa.fa_q8_read(lay, cache, k, k.clone())
    assert fa.fa_q8_poll_status(cache) == fa.FA_ERR_CAPACITY and (k[0] == -3).all() and (k[2] == -3).all() and (k[1] != -3).any()
    fa.fa_q8_step(lay, cache, q[:, 0].contiguous(), K[:, 0].contiguous(), K[:, 1].contiguous(), out[:, 0].contiguous(), ws)
    assert fa.fa_q8_poll_status(cache) == fa.FA_ERR_CAPACITY
    assert cache.state[:, 0].tolist() == [33, 32, -1]                       # (row 1 is full)
    fa.fa_q8_reset(lay, cache)
    assert (cache.state == 0).all() and fa.fa_q8_poll_status(cache) == fa.FA_OK


# ---- steps ------------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
@pytest.mark.parametrize("dtype,d,block", [("bf16", 128, 64), ("f32", 64, 16), ("bf16", 256, 128), ("bf16", 64, 32)])
def test_a_step_is_an_append_and_an_attention(fmt, dtype, d, block):
    """Bit for bit in the cache; results within the tolerance of the definition; rows of their own lengths, over ends of blocks, from empty ones on."""
    Hq, H = 4, 2
    lens = [0, block - 2, 2 * block - 1, 130]
    lens = lens + [7 * b % 40 for b in range(32 if dtype == "f32" else 0)]   # (more than 32 rows)
    B, steps = len(lens), 5
    lay, cache = make(B=B, Hq=Hq, H=H, d=d, block=block, nb=260 // block + 2, fmt=fmt, dtype=dtype)
    _, other = make(B=B, Hq=Hq, H=H, d=d, block=block, nb=260 // block + 2, fmt=fmt, dtype=dtype)
    most = max(lens)
    K, V = rand((B, most, H, d), dtype, 1), rand((B, most, H, d), dtype, 2)
    n = torch.tensor(lens, dtype=torch.int32, device="cuda")
    rows = ref.Rows(B, H, d, block, fmt, DT[dtype][0])
    for c in (cache, other):
        fa.fa_q8_write(lay, c, K, V, n)
    for b in range(B):
        rows.push(b, K[b, :lens[b]], V[b, :lens[b]])
    ws = fa.new_q8_workspace(lay)
    for i in range(steps):
        q, k, v = rand((B, Hq, d), dtype, 10 + i), rand((B, H, d), dtype, 20 + i), rand((B, H, d), dtype, 30 + i)
        out = torch.full_like(q, float("nan"))
        fa.fa_q8_step(lay, cache, q, k, v, out, ws)
        fa.fa_q8_append(lay, other, k[:, None], v[:, None])
        for b in range(B):
            rows.push(b, k[b:b + 1], v[b:b + 1])
        check_cache(lay, cache, rows, fmt)
        check_cache(lay, other, rows, fmt)
        assert (ws[:4096] == 0).all()
        for b in range(B):
            for h in range(H):
                G = Hq // H
                want, tol = ref.attention(rows.held("k", b, h), rows.held("v", b, h), q[b, None, h * G:(h + 1) * G].cpu().double(), 1, lay.softmax_scale, DT[dtype][0])
                assert ((out[b, None, h * G:(h + 1) * G].cpu().double() - want).abs() <= tol).all(), (i, b, h)


def test_steps_that_are_refused_attend_to_the_unchanged_row():
    B, Hq, H, d, block, nb = 3, 4, 2, 64, 16, 2
    lay, cache = make(B=B, Hq=Hq, H=H, d=d, block=block, nb=nb)
    K, V = rand((B, 32, H, d), "bf16", 1), rand((B, 32, H, d), "bf16", 2)
    lens = [32, 15, 15]                                                     # full; completes a block that has no page; goes ahead
    fa.fa_q8_write(lay, cache, K, V, torch.tensor(lens, dtype=torch.int32, device="cuda"))
    cache.block_table[1, 0] = -1
    rows = ref.Rows(B, H, d, block, "int8", torch.bfloat16)
    for b in range(B):
        rows.push(b, K[b, :lens[b]], V[b, :lens[b]])
    q, k, v = rand((B, Hq, d), "bf16", 3), rand((B, H, d), "bf16", 4), rand((B, H, d), "bf16", 5)
    out, ws = torch.empty_like(q), fa.new_q8_workspace(lay)
    fa.fa_q8_step(lay, cache, q, k, v, out, ws)
    assert fa.fa_q8_poll_status(cache) in (fa.FA_ERR_CAPACITY, fa.FA_ERR_INDEX)
    rows.push(2, k[2:], v[2:])
    assert cache.state[:, 0].tolist() == [32, 15, 16] and (cache.state[:, 1:] == 0).all() and (ws[:4096] == 0).all()
    check_cache(lay, cache, rows, "int8")
    for b in range(B):
        for h in range(H):
            want, tol = ref.attention(rows.held("k", b, h), rows.held("v", b, h), q[b, None, 2 * h:2 * h + 2].cpu().double(), 1, lay.softmax_scale, torch.bfloat16)
            assert ((out[b, None, 2 * h:2 * h + 2].cpu().double() - want).abs() <= tol).all(), (b, h)


def test_captured_steps_and_other_streams():
    """A graph of a step replayed while the row grows over a block's end, on a stream that is not the current one; results of
    the eager calls bit for bit."""
    B, Hq, H, d, block = 2, 8, 2, 128, 16
    lay, cache = make(B=B, Hq=Hq, H=H, d=d, block=block, nb=8)
    _, eager = make(B=B, Hq=Hq, H=H, d=d, block=block, nb=8)
    K, V = rand((B, 27, H, d), "bf16", 1), rand((B, 27, H, d), "bf16", 2)
    q, k, v = rand((B, Hq, d), "bf16", 3), rand((B, H, d), "bf16", 4), rand((B, H, d), "bf16", 5)
    out, want, ws, ws2 = torch.empty_like(q), torch.empty_like(q), fa.new_q8_workspace(lay), fa.new_q8_workspace(lay)
    fa.fa_q8_write(lay, eager, K, V)
    fa.fa_q8_step(lay, eager, q, k, v, want, ws2)                             # (the first call sets the kernels' attributes)
    fa.fa_q8_write(lay, eager, K, V)
    fa.fa_q8_write(lay, cache, K, V)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        fa.fa_q8_step(lay, cache, q, k, v, out, ws, stream=side)
    assert cache.state[:, 0].tolist() == [27, 27]
    for i in range(12):
        k.copy_(rand((B, H, d), "bf16", 50 + i))
        q.copy_(rand((B, Hq, d), "bf16", 80 + i))
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            graph.replay()
        torch.cuda.synchronize()
        fa.fa_q8_step(lay, eager, q, k, v, want, ws2)
        assert torch.equal(out, want), i
    assert cache.state[:, 0].tolist() == [39, 39]
    for n in ("k_tail", "v_tail", "state", "tail_amax", "k_scale", "v_scale"):
        assert torch.equal(getattr(cache, n), getattr(eager, n)), n


def test_a_request_through_the_operators_and_into_the_compressed_cache():
    """As a server would run it: the prompt in chunks with attention of each chunk, token steps, the cache read back, and its
    K and V handed to fa_compress; a decode step there agrees with the 8-bit cache's own attention where no dim is compressed."""
    B, Hq, H, d, block = 1, 8, 2, 128, 32
    n = 300
    lay, cache = make(B=B, Hq=Hq, H=H, d=d, block=block, nb=16, scale=0.09)
    K, V = rand((B, n, H, d), "bf16", 1, 0.0), rand((B, n, H, d), "bf16", 2, 0.0)
    rows = ref.Rows(B, H, d, block, "int8", torch.bfloat16)
    fa.fa_q8_reset(lay, cache)
    at = 0
    for chunk in (100, 1, 64, 130):
        k, v = K[:, at:at + chunk], V[:, at:at + chunk]
        fa.fa_q8_append(lay, cache, k, v)
        rows.push(0, k[0], v[0])
        attend_and_check(lay, cache, rows, rand((B, chunk, Hq, d), "bf16", at), "bf16")
        at += chunk
    ws = fa.new_q8_workspace(lay)
    out = torch.empty((B, Hq, d), dtype=torch.bfloat16, device="cuda")
    while at < n:
        q = rand((B, Hq, d), "bf16", 1000 + at)
        fa.fa_q8_step(lay, cache, q, K[:, at].contiguous(), V[:, at].contiguous(), out, ws)
        rows.push(0, K[0, at:at + 1], V[0, at:at + 1])
        at += 1
    check_cache(lay, cache, rows, "int8")
    k, v = torch.zeros_like(K), torch.zeros_like(V)
    fa.fa_q8_read(lay, cache, k, v)
    hybrid = fa.Layout(batch=B, n_q_heads=Hq, n_kv_heads=H, head_dim=d, n_full_k=d, n_full_v=d, n_coef=64, period=1024, l_init=4, l_local=64, max_mid=1024,
                       softmax_scale=0.09)
    every = torch.arange(d, dtype=torch.int32).expand(H, d)
    hc, hws = fa.Cache(hybrid, every, every), fa.new_workspace(hybrid)
    fa.fa_compress(hybrid, hc, k, v, hws)
    dense = torch.empty_like(out)
    fa.fa_decode_attention(hybrid, hc, q, dense, hws)
    assert fa.fa_poll_status(hc) == fa.FA_OK
    # the 8-bit side: its derived tolerance; the hybrid side: the 2e-2 of its own parity tests; K, V read back are within 2^-8
    # of what the cache holds, so the logits move by at most 2^-8 of sum |q k| (q, k unit normal) and the results by that share and 2^-8 of V
    for h in range(H):
        kk, vv, qq = rows.held("k", 0, h), rows.held("v", 0, h), q[0, None, 4 * h:4 * h + 4].cpu().double()
        want, tol = ref.attention(kk, vv, qq, 1, lay.softmax_scale, torch.bfloat16)
        assert ((out[0, None, 4 * h:4 * h + 4].cpu().double() - want).abs() <= tol).all()
        A = (qq[0].abs() @ kk.abs().T * 0.09).amax() * 2.0 ** -8
        mass = (torch.softmax(qq[0] @ kk.T * 0.09, -1) @ vv.abs())
        moved = 2 * torch.expm1(A) * mass + 2.0 ** -8 * mass
        assert ((dense[0, 4 * h:4 * h + 4].cpu().double() - want[0]).abs() <= 2e-2 + moved).all()

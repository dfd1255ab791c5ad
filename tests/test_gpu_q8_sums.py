"""fa_q8_attention over rows of millions of tokens, each summed by one CTA (all rows read the same pages): sums of one sign, where what a sum loses adds up."""
import math

import pytest
import torch

from paper_2506_11886_b200 import fa
from tests import q8_reference as ref
from tests.test_gpu_q8 import DT, FMT, make, rand

pytestmark = pytest.mark.gpu


def long_rows(K, V, B, Hq, d, n, dtype, fmt, scale):
    """B rows of n tokens that repeat the pages of K, V [1][held][1][d]."""
    block, held = 128, K.shape[1] // 128
    one, src = make(Hq=Hq, H=1, d=d, block=block, nb=held, fmt=fmt, dtype=dtype, extra=0, shuffle=False)
    fa.fa_q8_write(one, src, K, V)
    lay = fa.Q8Layout(batch=B, n_q_heads=Hq, n_kv_heads=1, head_dim=d, block=block, max_blocks=n // block, n_pages=held, format=FMT[fmt], kv_dtype=DT[dtype][1],
                      softmax_scale=scale)
    cache = fa.Q8Cache(lay)
    for name in ("k_pages", "v_pages", "k_scale", "v_scale"):
        getattr(cache, name).copy_(getattr(src, name))
    cache.block_table.copy_((torch.arange(n // block, dtype=torch.int32, device="cuda") % held).expand(B, -1))
    cache.state[:, 0] = n
    return lay, cache


@pytest.mark.parametrize("d,G,dtype", [(64, 1, "bf16"), (64, 10, "bf16"), (256, 1, "bf16"), (64, 1, "f32")])
def test_outputs_of_one_sign_over_sixteen_million_tokens(d, G, dtype):
    """q = 0: every weight is 1, an output the mean of its V.  A warp sums 131072 units of 16 tokens.  Counted for bf16: the output's half step, the weight's
    2^-11, the scale's product 2^-24, for cut-offs in runs of 1024 MMAs 2^-23 each of a sum that grows, 2^-14 in all, and as much for sums of 128 runs and all
    else that is rounded to 2^-24.
    For fp32: weights in two halves 2^-22, the MMAs of a unit 4 x 2^-23, the join and the division 25 x 2^-24, runs of 1024 additions and 128 of their sums,
    rounded by 2^-24 of a sum that grows, of either sign: six deviations of sqrt(1152 / 9) x 2^-24."""
    held, n = 256 * 128, 1 << 24
    V = (rand((1, held, 1, d), "f32", 1, 0.0).abs() + 0.25).to(DT[dtype][0])
    lay, cache = long_rows(V, V, 300, G, d, n, dtype, "int8", 0.125)
    q = torch.zeros((300, 1, G, d), dtype=DT[dtype][0], device="cuda")
    out = torch.full_like(q, math.nan)
    fa.fa_q8_attention(lay, cache, q, out, fa.new_q8_workspace(lay))
    assert fa.fa_q8_poll_status(cache) == fa.FA_OK
    want = (cache.v_pages.double().sum((1, 2)) * cache.v_scale.double()).mean(0) / 128
    err = float(((out.double() - want) / want).abs().max())
    if dtype == "bf16":
        assert err <= 2.0 ** -8 + 2.0 ** -11 + 2.0 ** -24 + 2.0 ** -14 + 2.0 ** -14
    else:
        assert err <= 2.0 ** -22 + 4 * 2.0 ** -23 + 25 * 2.0 ** -24 + 6 * math.sqrt(1152 / 9) * 2.0 ** -24


@pytest.mark.parametrize("G,n_q,B,dtype", [(1, 1, 300, "bf16"), (1, 1, 300, "f32"), (16, 5, 148, "bf16")])
def test_sums_of_equal_weights_over_sixteen_million_tokens(G, n_q, B, dtype):
    """Every key is the same and every value 1, so every output is 1 whatever p is; p = 0.70302 lies where sums rounded one way add up most: 8 p = 5.624 goes into a
    sum of 2^21 as 5.5.  Counted: the output's half step, the weights' 2^-11 (fp32 2^-22), V's scale 2^-24 (127 times it is 1 within that).  Sums of one sign: N
    equal additions rounded (cut off) one way are off by N 2^-24 (N 2^-23, of a sum that grows) at most.  The sum of p has runs of 1024 additions at most and 512
    runs: 2^-14 + 2^-15; the outputs of fp32 likewise, of bf16 2048 MMAs that cut off, 2^-13, and 512 runs."""
    d, n = 64, 1 << 24
    K = torch.ones((1, 256 * 128, 1, d), dtype=DT[dtype][0], device="cuda")
    lay, cache = long_rows(K, K, B, G, d, n, dtype, "int8", -math.log(0.70302))
    q = torch.full((B, n_q, G, d), -1.0 / 64, dtype=DT[dtype][0], device="cuda")
    out = torch.full_like(q, math.nan)
    fa.fa_q8_attention(lay, cache, q, out, fa.new_q8_workspace(lay, n_q))
    assert fa.fa_q8_poll_status(cache) == fa.FA_OK
    err = float((out.double() - 1).abs().max())
    sums = 2.0 ** -14 + 2.0 ** -15
    assert err <= (2.0 ** -8 + 2.0 ** -11 + 2.0 ** -24 + 2.0 ** -13 + 2.0 ** -15 + sums if dtype == "bf16" else 2.0 ** -22 + 2.0 ** -24 + 2 * sums), err


@pytest.mark.parametrize("dtype,fmt,d,G,n_q", [("bf16", "int8", 64, 1, 1), ("bf16", "e4m3", 64, 5, 2), ("f32", "int8", 64, 3, 1), ("bf16", "e4m3", 256, 1, 1)])
@pytest.mark.parametrize("order", [1, -1])
def test_runs_of_units_with_maxima_that_grow_or_not(dtype, fmt, d, G, n_q, order):
    """Three runs to a warp (a row of 300 000 tokens for each of 300 pairs): the scores' and the values' maxima grow from run to run, or are those of the first."""
    n, held = 300_032, 300_032
    K, V = rand((1, held, 1, d), dtype, 1, 0.0), rand((1, held, 1, d), dtype, 2, 0.0)
    ramp = torch.linspace(0.05, 1.0, held, device="cuda")[None, :, None, None]
    steps = (torch.arange(held, device="cuda") // 40_000)[None, :, None, None]
    K, V = (K.float() * ramp).to(DT[dtype][0]), (V.float() * torch.exp2(steps - 4.0)).to(DT[dtype][0])
    if order < 0:
        K, V = K.flip(1).contiguous(), V.flip(1).contiguous()
    lay, cache = long_rows(K, V, 300, G, d, n, dtype, fmt, 8.0 / d)
    rows = ref.Rows(1, 1, d, 128, fmt, DT[dtype][0])
    rows.push(0, K[0], V[0])
    k, v = rows.held("k", 0, 0), rows.held("v", 0, 0)
    q = rand((300, n_q, G, d), dtype, 3, 0.0)
    out = torch.full_like(q, math.nan)
    fa.fa_q8_attention(lay, cache, q, out, fa.new_q8_workspace(lay, n_q))
    assert fa.fa_q8_poll_status(cache) == fa.FA_OK
    assert torch.isfinite(out.float()).all()
    for b in (0, 1, 73, 147, 148, 222, 299):
        want, tol = ref.attention(k, v, q[b].cpu().double(), n_q, lay.softmax_scale, DT[dtype][0])
        err = (out[b].cpu().double() - want).abs()
        assert (err <= tol).all(), (b, float((err / tol).max()))

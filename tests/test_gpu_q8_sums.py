"""fa_q8_attention over rows of millions of tokens, each summed by one CTA (all rows read the same pages): sums of one sign, where what a sum loses adds up."""
import math

import pytest
import torch

from paper_2506_11886_b200 import fa
from tests.test_gpu_q8 import FMT, DT, make, rand

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


@pytest.mark.parametrize("G,n_q,B,dtype", [(1, 1, 300, "f32"), (16, 5, 148, "bf16")])
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

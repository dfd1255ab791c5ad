"""fa_q8_attention where V lies near the ends of the number range: what counts in a row has V scales down to the smallest numbers, or scales
that differ by as many powers of two as the scores differ the other way.  Tolerances are relative to V (tests/q8_reference.py adds 1e-30 to its own)."""
import math

import pytest
import torch

from paper_2506_11886_b200 import fa
from tests import q8_reference as ref
from tests.test_gpu_q8 import DT, make, rand

pytestmark = pytest.mark.gpu


def attend_and_check(lay, cache, rows, q, fmt, dtype):
    """The reference's tolerance for V times 2^100, which makes nothing of its 1e-30; and
      * the output's smallest step (half of it; bf16 comes from fp32 results that have one of their own);
      * weights are halves (of two, in fp32) that are whole multiples of 2^-24, so off by 2^-25 each.  The reference counts that against a largest weight
        of 2^13 or more; where V scales are below 2^-111, a weight is p times the scale times 2^126 instead.  A V code is at most `top`: 2^-25 top 2^-126 / l
        a token in the result, l the sum of p = 2^(score - the maximum's next whole number)."""
    n_q, G = q.shape[1], lay.n_q_heads // lay.n_kv_heads
    out = torch.full_like(q, math.nan)
    fa.fa_q8_attention(lay, cache, q, out, fa.new_q8_workspace(lay, n_q))
    assert fa.fa_q8_poll_status(cache) == fa.FA_OK
    got, step = out.cpu().double(), 2.0 ** -134 + 2.0 ** -147 if dtype == "bf16" else 2.0 ** -149
    for b in range(lay.batch):
        for h in range(lay.n_kv_heads):
            k, v, qq = rows.held("k", b, h), rows.held("v", b, h), q[b, :, h * G:(h + 1) * G].cpu().double()
            want, tol = ref.attention(k, v * 2.0 ** 100, qq, n_q, lay.softmax_scale, DT[dtype][0])
            tol = tol * 2.0 ** -100 + step
            for i in range(n_q):
                seen = k.shape[0] - n_q + i + 1
                if seen > 0:
                    s = qq[i] @ k[:seen].T * (lay.softmax_scale / math.log(2.0))
                    l = torch.exp2(s - torch.ceil(s.amax(-1, keepdim=True))).sum(-1)
                    tol[i] += (seen * 2.0 ** -151 * ref.TOP[fmt] / l)[:, None]
            err = (got[b, :, h * G:(h + 1) * G] - want * 2.0 ** -100).abs()
            assert (err <= tol).all(), (b, h, float((err / tol).max()), float(err.max()), float(want.abs().max() * 2.0 ** -100))


@pytest.mark.parametrize("size", [1e-30, 1e-33, 1e-36, 1e-39])
@pytest.mark.parametrize("n_q", [1, 40])
@pytest.mark.parametrize("fmt,dtype,d", [("int8", "bf16", 128), ("e4m3", "bf16", 64), ("int8", "f32", 64), ("e4m3", "f32", 256)])
def test_all_of_v_is_small(fmt, dtype, d, n_q, size):
    """Rows without a token, of a tail, of pages, of both, in several parts."""
    Hq, H, block, lens = 8, 2, 32, [0, 5, 64, 100, 700]
    B, most = len(lens), 704
    lay, cache = make(B=B, Hq=Hq, H=H, d=d, block=block, nb=most // block, fmt=fmt, dtype=dtype)
    K, V = rand((B, most, H, d), dtype, 1), (rand((B, most, H, d), "f32", 2) * size).to(DT[dtype][0])
    fa.fa_q8_write(lay, cache, K, V, torch.tensor(lens, dtype=torch.int32, device="cuda"))
    rows = ref.Rows(B, H, d, block, fmt, DT[dtype][0])
    for b in range(B):
        rows.push(b, K[b, :lens[b]], V[b, :lens[b]])
    attend_and_check(lay, cache, rows, rand((B, n_q, Hq, d), dtype, 3), fmt, dtype)


@pytest.mark.parametrize("apart", [50, 112, 115, 120])
@pytest.mark.parametrize("n_q", [1, 40])
@pytest.mark.parametrize("fmt,dtype", [("int8", "bf16"), ("e4m3", "bf16"), ("int8", "f32"), ("e4m3", "f32")])
def test_v_scales_and_scores_apart_the_other_way(fmt, dtype, n_q, apart):
    """Every other block (and the tail of one of the rows) has scores `apart` powers of two lower and V as much larger: both sorts count alike."""
    Hq, H, d, block, lens = 4, 1, 64, 16, [200, 217, 201]
    lay, cache = make(B=3, Hq=Hq, H=H, d=d, block=block, nb=14, fmt=fmt, dtype=dtype, scale=math.log(2.0) / 32)
    odd = (torch.arange(217) // block % 2)[None, :, None, None]
    low = torch.cat((odd, 1 - odd, odd))                               # rows 0 and 2 begin with the small V, row 1 with the large
    # a key of a everywhere against q = 0.5: 64 a / 2 / 32 = a powers of two
    K = torch.where(low == 1, -apart / 2, apart / 2) * torch.ones(3, 217, H, d)
    V = rand((3, 217, H, d), "f32", 2, 0.0).cpu() * torch.exp2(torch.where(low == 1, apart - 60.0, -60.0))
    K, V = K.to(DT[dtype][0]).cuda(), V.to(DT[dtype][0]).cuda()
    fa.fa_q8_write(lay, cache, K, V, torch.tensor(lens, dtype=torch.int32, device="cuda"))
    rows = ref.Rows(3, H, d, block, fmt, DT[dtype][0])
    for b in range(3):
        rows.push(b, K[b, :lens[b]], V[b, :lens[b]])
    attend_and_check(lay, cache, rows, torch.full((3, n_q, Hq, d), 0.5, dtype=DT[dtype][0], device="cuda"), fmt, dtype)

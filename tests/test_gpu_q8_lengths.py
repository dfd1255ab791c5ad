"""fa_q8_attention on rows whose length in `state` is none, with few columns to a KV head and with many."""
import math

import pytest
import torch

from paper_2506_11886_b200 import fa
from tests.test_gpu_q8 import make, rand

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("n_q", [1, 16, 17, 300])
@pytest.mark.parametrize("bad", [(33, 32, -1), (32, 33, 32), (32, 32, -2 ** 31)])
def test_a_length_that_is_none_is_reported_whatever_the_number_of_queries(n_q, bad):
    """4 query heads to a KV head: 4, 64, 68 and 1200 columns."""
    lay, cache = make(B=3, H=2, d=64, block=16, nb=2)
    K = rand((3, 32, 2, 64), "bf16", 1)
    fa.fa_q8_write(lay, cache, K, K)
    q, ws = rand((3, n_q, 8, 64), "bf16", 2), fa.new_q8_workspace(lay, n_q)
    good = torch.full_like(q, math.nan)
    fa.fa_q8_attention(lay, cache, q, good, ws)
    assert fa.fa_q8_poll_status(cache) == fa.FA_OK
    cache.state[:, 0] = torch.tensor(bad, dtype=torch.int32)
    out = torch.full_like(q, math.nan)
    fa.fa_q8_attention(lay, cache, q, out, ws)
    assert fa.fa_q8_poll_status(cache) == fa.FA_ERR_CAPACITY
    for b, n in enumerate(bad):
        if n == 32:
            # (the rows' work is cut another way now: fp32 sums in another order, so a step of bf16 at most)
            assert ((out[b].float() - good[b].float()).abs() <= 2.0 ** -7 * good[b].float().abs() + 1e-6).all()
        else:
            assert (out[b] == 0).all()

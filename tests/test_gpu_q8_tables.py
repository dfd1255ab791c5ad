"""Block tables that are much longer than the rows."""
import math

import pytest
import torch

from paper_2506_11886_b200 import fa
from tests.test_gpu_q8 import make, rand

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("B,Hq,H,d,block,nb,n_q", [(16, 32, 8, 128, 128, 8192, 2048), (2, 16, 4, 64, 16, 1 << 24, 65)])
def test_tables_of_a_million_tokens_and_more(B, Hq, H, d, block, nb, n_q):
    """What a row could hold has no effect on the results: those of a table that just fits, bit for bit."""
    lens = [(401 * b) % 1500 if b else 1777 for b in range(B)]
    short = -(-max(lens) // block)
    lay, cache = make(B=B, Hq=Hq, H=H, d=d, block=block, nb=short)
    K = rand((B, max(lens), H, d), "bf16", 1)
    fa.fa_q8_write(lay, cache, K, K.flip(1), torch.tensor(lens, dtype=torch.int32, device="cuda"))
    long = fa.Q8Layout(batch=B, n_q_heads=Hq, n_kv_heads=H, head_dim=d, block=block, max_blocks=nb, n_pages=lay.n_pages, softmax_scale=lay.softmax_scale)
    table = torch.full((B, nb), -1, dtype=torch.int32, device="cuda")
    table[:, :short] = cache.block_table
    other = fa.Q8Cache(long, buffers={n: getattr(cache, n) for n in ("k_pages", "v_pages", "k_scale", "v_scale", "k_tail", "v_tail", "tail_amax", "state")} | {"block_table": table})
    q = rand((B, n_q, Hq, d), "bf16", 2)
    want, out = torch.full_like(q, math.nan), torch.full_like(q, math.nan)
    fa.fa_q8_attention(lay, cache, q, want, fa.new_q8_workspace(lay, n_q))
    fa.fa_q8_attention(long, other, q, out, fa.new_q8_workspace(long, n_q))
    assert fa.fa_q8_poll_status(cache) == fa.FA_OK and fa.fa_q8_poll_status(other) == fa.FA_OK
    assert torch.equal(want, out) and torch.isfinite(out.float()).all()

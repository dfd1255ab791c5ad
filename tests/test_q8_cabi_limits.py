"""Sizes that only one of the two attention kernels can count: host logic only, nothing is launched."""
import ctypes as C

import pytest

from paper_2506_11886_b200 import build, fa


@pytest.fixture(scope="module", autouse=True)
def _built():
    build.build_library()


def _call(n_q, ws_bytes, **kw):
    base = dict(batch=16, n_q_heads=32, n_kv_heads=8, head_dim=128, block=128, max_blocks=8192, n_pages=1024, format=fa.FA_Q8_INT8, kv_dtype=fa.FA_BF16,
                softmax_scale=0.1)
    base.update(kw)
    lay = fa.Q8Layout(**base).c()
    cache = fa.fa_q8_cache(*[16 * (i + 1) for i in range(len(fa._Q8_FIELDS))])       # never looked at
    return fa.lib().fa_q8_attention(C.byref(lay), C.byref(cache), 16, 0, 32 * lay.head_dim, lay.head_dim, 16, n_q, 16, ws_bytes, None)


def test_chunks_over_long_block_tables():
    """16 rows, tables of a million tokens, 2048 queries: 2^32 pieces of 16 columns and 16 tokens, 2^25 of 256 columns and 128 tokens.  The call goes
    on to the check of its workspace (which is refused here)."""
    need = fa.fa_q8_workspace_bytes(fa.Q8Layout(batch=16, n_q_heads=32, n_kv_heads=8, head_dim=128, block=128, max_blocks=8192, n_pages=1024, softmax_scale=0.1), 2048)
    assert _call(2048, need - 1) == fa.FA_ERR_WORKSPACE
    assert _call(2048, 4096, head_dim=64) == fa.FA_ERR_WORKSPACE
    # these go by 16 columns
    assert _call(2048, 1 << 40, kv_dtype=fa.FA_F32) == fa.FA_ERR_UNSUPPORTED
    assert _call(2048, 1 << 40, head_dim=256) == fa.FA_ERR_UNSUPPORTED
    # more than either counts
    assert _call(2048, 1 << 40, batch=8192) == fa.FA_ERR_UNSUPPORTED
    # a few queries of the same rows
    assert _call(16, 4096) == fa.FA_ERR_WORKSPACE


@pytest.mark.parametrize("tokens", [4096, 131072, 131072 + 128, 1 << 20, 1 << 24])
@pytest.mark.parametrize("B,Hq,H,d", [(1, 32, 8, 128), (300, 1, 1, 64), (40, 80, 8, 256), (2, 8, 8, 64), (1, 4, 1, 256)])
def test_a_workspace_serves_fewer_queries_too(tokens, B, Hq, H, d):
    lay = fa.Q8Layout(batch=B, n_q_heads=Hq, n_kv_heads=H, head_dim=d, block=128, max_blocks=tokens // 128, n_pages=8)
    sizes = [fa.fa_q8_workspace_bytes(lay, n) for n in (1, 2, 3, 5, 8, 9, 16, 17, 40, 64, 65, 300)]
    assert sizes == sorted(sizes) and sizes[-1] < 256 << 20

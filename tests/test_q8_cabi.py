"""Refusals and sizes of the dense cache in 8 bits: host logic only, nothing is launched."""
import ctypes as C

import pytest
import torch

from paper_2506_11886_b200 import build, fa


@pytest.fixture(scope="module", autouse=True)
def _built():
    build.build_library()


def _layout(**kw):
    base = dict(batch=2, n_q_heads=32, n_kv_heads=8, head_dim=128, block=64, max_blocks=512, n_pages=1024, format=fa.FA_Q8_INT8, kv_dtype=fa.FA_BF16,
                softmax_scale=0.1)
    base.update(kw)
    return fa.Q8Layout(**base)


def _cache(**kw):
    c = fa.fa_q8_cache(*[16 * (i + 1) for i in range(len(fa._Q8_FIELDS))])       # never looked at
    for n, v in kw.items():
        setattr(c, n, v)
    return c


def test_struct_layouts():
    assert C.sizeof(fa.fa_q8_layout) == 10 * 4
    assert C.sizeof(fa.fa_q8_cache) == 10 * C.sizeof(C.c_void_p)


def test_sizes():
    sz = fa.fa_q8_cache_sizes_of(_layout())
    assert sz["k_pages"] == sz["v_pages"] == 1024 * 8 * 64 * 128 and sz["k_scale"] == 1024 * 8 * 4
    assert sz["k_tail"] == 2 * 8 * 64 * 128 * 2 and sz["tail_amax"] == 2 * 8 * 2 * 4
    assert sz["block_table"] == 2 * 512 * 4 and sz["state"] == 2 * 16 and sz["status"] == 16
    assert fa.fa_q8_cache_sizes_of(_layout(kv_dtype=fa.FA_F32))["k_tail"] == 2 * sz["k_tail"]
    big = fa.fa_q8_cache_sizes_of(_layout(n_pages=1 << 20))                        # past 32 bits
    assert big["k_pages"] == (1 << 20) * 8 * 64 * 128
    one, many = fa.fa_q8_workspace_bytes(_layout()), fa.fa_q8_workspace_bytes(_layout(), 64)
    assert 4096 < one <= many


@pytest.mark.parametrize("kw,status", [
    (dict(batch=0), fa.FA_ERR_INVALID_ARG), (dict(n_kv_heads=5), fa.FA_ERR_INVALID_ARG), (dict(max_blocks=0), fa.FA_ERR_INVALID_ARG),
    (dict(n_pages=-1), fa.FA_ERR_INVALID_ARG), (dict(format=2), fa.FA_ERR_INVALID_ARG), (dict(kv_dtype=2), fa.FA_ERR_INVALID_ARG),
    (dict(softmax_scale=0.0), fa.FA_ERR_INVALID_ARG), (dict(softmax_scale=float("nan")), fa.FA_ERR_INVALID_ARG),
    (dict(head_dim=96), fa.FA_ERR_UNSUPPORTED), (dict(head_dim=512), fa.FA_ERR_UNSUPPORTED), (dict(block=48), fa.FA_ERR_UNSUPPORTED),
    (dict(block=256), fa.FA_ERR_UNSUPPORTED), (dict(n_q_heads=8 * 17), fa.FA_ERR_UNSUPPORTED), (dict(batch=65536), fa.FA_ERR_UNSUPPORTED),
    (dict(max_blocks=1 << 25), fa.FA_ERR_UNSUPPORTED),
])
def test_bad_layouts(kw, status):
    with pytest.raises(fa.FaError) as e:
        fa.fa_q8_cache_sizes_of(_layout(**kw))
    assert e.value.status == status
    lay, c, lib = _layout(**kw).c(), _cache(), fa.lib()
    assert lib.fa_q8_write(C.byref(lay), C.byref(c), 16, 16, 0, 1024, 128, 4, None, None) == status
    assert lib.fa_q8_append(C.byref(lay), C.byref(c), 16, 16, 0, 1024, 128, 4, None, None) == status
    assert lib.fa_q8_read(C.byref(lay), C.byref(c), 16, 16, 0, 1024, 128, 0, 4, None) == status
    assert lib.fa_q8_attention(C.byref(lay), C.byref(c), 16, 0, 4096, 128, 16, 1, 16, 1 << 30, None) == status
    assert lib.fa_q8_step(C.byref(lay), C.byref(c), 16, 16, 16, 16, 16, 1 << 30, None) == status
    assert lib.fa_q8_reset(C.byref(lay), C.byref(c), None) == status


def test_bad_arguments():
    lib, lay = fa.lib(), _layout().c()
    bad, ok = fa.FA_ERR_INVALID_ARG, _cache()
    for n in fa._Q8_FIELDS:
        for v in (0, 24):                                                          # missing, not on 16 bytes
            c = _cache(**{n: v})
            assert lib.fa_q8_write(C.byref(lay), C.byref(c), 16, 16, 0, 1024, 128, 4, None, None) == bad, (n, v)
            assert lib.fa_q8_attention(C.byref(lay), C.byref(c), 16, 0, 4096, 128, 16, 1, 16, 1 << 30, None) == bad, (n, v)
    for K, V, sb, st, sh, n in ((0, 16, 0, 1024, 128, 4), (16, 0, 0, 1024, 128, 4), (24, 16, 0, 1024, 128, 4), (16, 24, 0, 1024, 128, 4), (16, 16, -8, 1024, 128, 4),
                                (16, 16, 0, 120, 128, 4), (16, 16, 0, 1024, 120, 4), (16, 16, 0, 1028, 128, 4), (16, 16, 4, 1024, 128, 4), (16, 16, 0, 1024, 128, -1)):
        assert lib.fa_q8_write(C.byref(lay), C.byref(ok), K, V, sb, st, sh, n, None, None) == bad
        assert lib.fa_q8_append(C.byref(lay), C.byref(ok), K, V, sb, st, sh, n, None, None) == bad
        assert lib.fa_q8_read(C.byref(lay), C.byref(ok), K, V, sb, st, sh, 0, n, None) == bad
    assert lib.fa_q8_read(C.byref(lay), C.byref(ok), 16, 16, 0, 1024, 128, -1, 4, None) == bad
    assert lib.fa_q8_read(C.byref(lay), C.byref(ok), 16, 16, 0, 1024, 128, 0x7fffffff, 4, None) == bad
    assert lib.fa_q8_append(C.byref(lay), C.byref(ok), None, None, 0, 0, 0, 0, None, None) == fa.FA_OK          # no tokens: nothing to do
    assert lib.fa_q8_read(C.byref(lay), C.byref(ok), 16, 16, 0, 1024, 128, 512 * 64, 4, None) == fa.FA_OK       # behind what a row can hold
    wide = _layout(batch=65535, n_kv_heads=4096, n_q_heads=4096).c()                                            # more blocks than a launch counts
    assert lib.fa_q8_write(C.byref(wide), C.byref(ok), 16, 16, 0, 1024, 128, 1 << 20, None, None) == fa.FA_ERR_UNSUPPORTED
    assert lib.fa_q8_read(C.byref(lay), C.byref(ok), None, None, 0, 0, 0, 5, 0, None) == fa.FA_OK

    def attend(q=16, sb=0, si=4096, sg=128, out=16, n_q=1, ws=16, size=1 << 30):
        return lib.fa_q8_attention(C.byref(lay), C.byref(ok), q, sb, si, sg, out, n_q, ws, size, None)

    assert attend(q=0) == attend(out=0) == attend(q=24) == attend(out=8) == attend(sb=-8) == attend(si=120) == attend(sg=64) == attend(sg=132) == bad
    assert attend(n_q=-1) == bad and attend(n_q=0) == fa.FA_OK and attend(n_q=1 << 22) == fa.FA_ERR_UNSUPPORTED
    need = fa.fa_q8_workspace_bytes(_layout())
    assert attend(ws=0) == attend(ws=24) == attend(size=need - 1) == fa.FA_ERR_WORKSPACE
    step = lambda q=16, k=16, v=16, o=16, ws=16, size=1 << 30: lib.fa_q8_step(C.byref(lay), C.byref(ok), q, k, v, o, ws, size, None)
    assert step(q=0) == step(k=0) == step(v=0) == step(o=0) == step(k=24) == step(v=8) == bad
    assert step(ws=0) == step(size=need - 1) == fa.FA_ERR_WORKSPACE
    assert lib.fa_q8_workspace_bytes(C.byref(lay), 0, C.byref(C.c_size_t())) == bad and lib.fa_q8_workspace_bytes(C.byref(lay), 1, None) == bad
    assert lib.fa_q8_poll_status(None, None) == bad and lib.fa_q8_cache_sizes_of(C.byref(lay), None) == bad


def test_the_binding_checks_its_tensors():
    lay = _layout(batch=1, n_pages=4, max_blocks=4)
    with pytest.raises(ValueError):
        fa.Q8Cache(lay, buffers=dict(pages=torch.zeros(1)), device="cpu")
    with pytest.raises(ValueError):
        fa.Q8Cache(lay, buffers=dict(k_scale=torch.zeros(4, 7)), device="cpu")
    c = fa.Q8Cache(lay, device="cpu")
    assert c.block_table.tolist() == [[0, 1, 2, 3]] and c.k_pages.dtype == torch.int8 and c.k_pages.shape == (4, 8, 64, 128)
    assert fa.Q8Cache(_layout(batch=2, n_pages=5, max_blocks=4), device="cpu").block_table.tolist() == [[0, 1, 2, 3], [4, -1, -1, -1]]
    K = torch.zeros(1, 4, 8, 128, dtype=torch.bfloat16)
    for call in (lambda: fa.fa_q8_write(lay, c, K, K), lambda: fa.fa_q8_append(lay, c, K, K), lambda: fa.fa_q8_read(lay, c, K, K),
                 lambda: fa.fa_q8_attention(lay, c, torch.zeros(1, 32, 128), torch.zeros(1, 32, 128), K),
                 lambda: fa.fa_q8_step(lay, c, K, K, K, K, K)):
        with pytest.raises(ValueError):
            call()

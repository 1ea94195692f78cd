"""CPU-side checks of the 8-bit calls: what they refuse on the host, before any launch.  No kernel runs here."""
import ctypes

import pytest


@pytest.fixture(scope="module")
def L():
    from paper_2512_15176_b200 import build
    build.build()
    from paper_2512_15176_b200 import binding
    binding.lib()
    return binding


def _desc(L, D=128):
    fake = 0x1000
    return L.deer_kv_desc(fake, fake, fake, fake, fake, fake, fake, fake, 4, 2, D, 16, 1, 4)


@pytest.fixture()
def handles(L):
    lib = L.lib()
    fake = 0x1000
    plain, quant = ctypes.c_void_p(), ctypes.c_void_p()
    d = _desc(L)
    q = L.deer_kv_quant_desc(fake, fake, fake, fake)
    assert lib.deer_kv_create(ctypes.byref(plain), ctypes.byref(d)) == L.DEER_OK
    assert lib.deer_kv_create_quant(ctypes.byref(quant), ctypes.byref(d), ctypes.byref(q)) == L.DEER_OK
    yield plain, quant
    lib.deer_kv_destroy(plain)
    lib.deer_kv_destroy(quant)


def test_create_refusals(L):
    lib, fake = L.lib(), 0x1000
    kv, d = ctypes.c_void_p(), _desc(L)
    ok = L.deer_kv_quant_desc(fake, fake, fake, fake)
    assert lib.deer_kv_create_quant(ctypes.byref(kv), ctypes.byref(d), None) == L.DEER_ERR_INVALID_ARG
    for i in range(4):
        q = L.deer_kv_quant_desc(*[0 if j == i else fake for j in range(4)])
        assert lib.deer_kv_create_quant(ctypes.byref(kv), ctypes.byref(d), ctypes.byref(q)) == L.DEER_ERR_INVALID_ARG
    q = L.deer_kv_quant_desc(fake, fake, fake + 8, fake)
    assert lib.deer_kv_create_quant(ctypes.byref(kv), ctypes.byref(d), ctypes.byref(q)) == L.DEER_ERR_INVALID_ARG
    bad = _desc(L, 96)
    assert lib.deer_kv_create_quant(ctypes.byref(kv), ctypes.byref(bad), ctypes.byref(ok)) == L.DEER_ERR_UNSUPPORTED


def test_each_cache_kind_is_refused_by_the_other_kinds_calls(L, handles):
    lib, f = L.lib(), 0x1000
    plain, quant = handles
    assert lib.deer_block_attn(quant, f, f, f, f, f, 1, 8, 4, 0, 0, 1.0, 64, f, 1 << 20, None) == L.DEER_ERR_UNSUPPORTED
    assert lib.deer_block_attn_rows(quant, f, f, f, f, f, f, 1, 8, 4, 1, 0, 1.0, 64, f, 1 << 20, None) == L.DEER_ERR_UNSUPPORTED
    assert lib.deer_block_attn_quant(plain, f, f, f, f, f, None, 1, 8, 4, 0, 1.0, 64, f, 1 << 20, None) == L.DEER_ERR_UNSUPPORTED
    assert lib.deer_kv_store(plain, f, f, f, f, 1, 8, None) == L.DEER_ERR_UNSUPPORTED
    dev = L.deer_step_dev()
    assert lib.deer_verify_step_host(quant, ctypes.byref(dev), f, f, f, f, f, f, 1, 8, 4, 512, 1000, 1.0, 64, f, f, f, None) == L.DEER_ERR_UNSUPPORTED


def test_attention_and_store_refusals(L, handles):
    lib, f = L.lib(), 0x1000
    _, kv = handles
    call = lambda **a: lib.deer_block_attn_quant(kv, *[a.get(n, d) for n, d in (
        ("ids", f), ("q", f), ("k_blk", f), ("v_blk", f), ("out", f), ("states", None), ("B", 1), ("k", 8), ("Hq", 4), ("mask", 0),
        ("scale", 1.0), ("max_len", 64), ("ws", f), ("ws_bytes", 1 << 24), ("stream", None))])
    for n in ("ids", "q", "k_blk", "v_blk", "out"):
        assert call(**{n: None}) == L.DEER_ERR_INVALID_ARG
    for n in ("q", "k_blk", "v_blk", "out", "ws"):
        assert call(**{n: f + 2}) == L.DEER_ERR_INVALID_ARG
    assert call(k=33) == L.DEER_ERR_UNSUPPORTED and call(k=0) == L.DEER_ERR_UNSUPPORTED
    assert call(B=-1) == L.DEER_ERR_UNSUPPORTED
    assert call(Hq=3) == L.DEER_ERR_INVALID_ARG and call(Hq=0) == L.DEER_ERR_INVALID_ARG
    assert call(mask=2) == L.DEER_ERR_INVALID_ARG
    assert call(states=f) == L.DEER_ERR_INVALID_ARG                     # row states belong to the bidirectional mask
    assert call(max_len=-1) == L.DEER_ERR_INVALID_ARG
    need = lib.deer_block_attn_quant_workspace_bytes(1, 8, 4, 2, 128, 100000)
    assert need > 0
    assert call(max_len=100000, ws_bytes=need - 1) == L.DEER_ERR_WORKSPACE
    assert call(max_len=100000, ws=None, ws_bytes=need) == L.DEER_ERR_WORKSPACE
    assert call(B=0, ws=None, ws_bytes=0) == L.DEER_OK
    assert lib.deer_block_attn_quant_workspace_bytes(0, 8, 4, 2, 128, 64) == 0
    assert lib.deer_block_attn_quant_workspace_bytes(1, 8, 5, 2, 128, 64) == 0
    assert lib.deer_kv_store(kv, None, f, f, f, 1, 8, None) == L.DEER_ERR_INVALID_ARG
    assert lib.deer_kv_store(kv, f, f + 4, f, f, 1, 8, None) == L.DEER_ERR_INVALID_ARG
    assert lib.deer_kv_store(kv, f, f, f, f, 1, -1, None) == L.DEER_ERR_UNSUPPORTED
    assert lib.deer_kv_store(kv, f, f, f, f, 1, (1 << 24) + 1, None) == L.DEER_ERR_UNSUPPORTED
    assert lib.deer_kv_store(kv, f, f, f, f, 0, 8, None) == L.DEER_OK
    assert lib.deer_kv_store(kv, f, f, f, None, 1, 0, None) == L.DEER_OK
    assert lib.deer_kv_reserve_rows(kv, f, 1025, 8, None) == L.DEER_ERR_UNSUPPORTED
    assert lib.deer_kv_reserve_rows(kv, f, 1, (1 << 24) + 1, None) == L.DEER_ERR_UNSUPPORTED
    assert lib.deer_kv_commit_rows(kv, f, f, 1, -1, None) == L.DEER_ERR_UNSUPPORTED
    assert lib.deer_kv_reserve_rows(kv, f, 0, 4096, None) == L.DEER_OK
    # the block-sized calls keep their limit
    assert lib.deer_kv_reserve(kv, f, 1, 33, None) == L.DEER_ERR_UNSUPPORTED
    assert lib.deer_kv_commit(kv, f, f, 1, 33, None) == L.DEER_ERR_UNSUPPORTED


def test_row_wise_and_linear_refusals(L):
    lib, f = L.lib(), 0x1000
    assert lib.deer_rmsnorm_quant(None, None, f, None, f, f, 4, 128, 1e-6, None) == L.DEER_ERR_INVALID_ARG
    assert lib.deer_rmsnorm_quant(f, None, None, None, f, f, 4, 128, 1e-6, None) == L.DEER_ERR_INVALID_ARG
    assert lib.deer_rmsnorm_quant(f, f + 2, f, None, f, f, 4, 128, 1e-6, None) == L.DEER_ERR_INVALID_ARG
    assert lib.deer_rmsnorm_quant(f, None, f, None, f, f, -1, 128, 1e-6, None) == L.DEER_ERR_INVALID_ARG
    for hid in (0, 100, 65552):
        assert lib.deer_rmsnorm_quant(f, None, f, None, f, f, 4, hid, 1e-6, None) == L.DEER_ERR_UNSUPPORTED
    assert lib.deer_rmsnorm_quant(f, None, f, None, f, f, 0, 128, 1e-6, None) == L.DEER_OK
    assert lib.deer_quantize(f, 0, None, f, 4, 128, None) == L.DEER_ERR_INVALID_ARG
    assert lib.deer_quantize(f, 0, f, f + 2, 4, 128, None) == L.DEER_ERR_INVALID_ARG
    assert lib.deer_quantize(f, 1, f, f, 4, 100, None) == L.DEER_ERR_UNSUPPORTED
    assert lib.deer_quantize(f, 1, f, f, 0, 128, None) == L.DEER_OK
    assert lib.deer_linear_quant(f, f, f, None, None, f, 4, 128, 128, None) == L.DEER_ERR_INVALID_ARG
    assert lib.deer_linear_quant(f, f, f + 8, f, None, f, 4, 128, 128, None) == L.DEER_ERR_INVALID_ARG
    assert lib.deer_linear_quant(f, f, f, f, None, f, -4, 128, 128, None) == L.DEER_ERR_INVALID_ARG
    for K, N in ((100, 128), (128, 100), (0, 128), (128, 8)):
        assert lib.deer_linear_quant(f, f, f, f, None, f, 4, K, N, None) == L.DEER_ERR_UNSUPPORTED
    assert lib.deer_linear_quant(f, f, f, f, None, f, 0, 128, 128, None) == L.DEER_OK


def test_linear_refuses_sizes_whose_indices_would_not_fit(L):
    lib, f = L.lib(), 0x1000
    big = (1 << 30) + 16
    for M, K, N in ((big, 128, 128), (4, big, 128), (4, 128, big)):
        assert lib.deer_linear_quant(f, f, f, f, None, f, M, K, N, None) == L.DEER_ERR_UNSUPPORTED

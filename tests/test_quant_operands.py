"""What the 8-bit calls of the binding refuse before the library sees a pointer: operands of another type or size than the
call would read or write.  Host tensors; no kernel runs here."""
import pytest
import torch

BF, F32, F8, I32 = torch.bfloat16, torch.float32, torch.float8_e4m3fn, torch.int32


@pytest.fixture(scope="module")
def L():
    from paper_2512_15176_b200 import build
    build.build()
    from paper_2512_15176_b200 import binding
    binding.lib()
    return binding


def z(*shape, dtype=BF):
    return torch.zeros(*shape, dtype=dtype)


def _refused(L, call, good, bad):
    """`bad`: operand name -> tensors that must be refused in its place."""
    for name, values in bad.items():
        for v in values:
            with pytest.raises(L.DeerError) as e:
                call(**{**good, name: v})
            assert e.value.code == L.DEER_ERR_INVALID_ARG, (name, str(e.value))


def test_rmsnorm_operands(L):
    good = dict(x=z(3, 272), gamma=z(272), codes=z(3, 272, dtype=F8), scales=z(3, 3, dtype=F32), eps=1e-6, residual=z(3, 272), total=z(3, 272))
    _refused(L, L.deer_rmsnorm_quant, good, dict(
        x=[z(3, 272, dtype=F32), z(3, 288)], gamma=[z(256), z(272, dtype=F32)], codes=[z(3, 272), z(2, 272, dtype=F8)],
        scales=[z(3, 2, dtype=F32), z(3, 3)], residual=[z(2, 272), z(3, 272, dtype=F32)], total=[z(3, 256), z(3, 272, dtype=F32)]))


def test_quantize_operands(L):
    good = dict(x=z(3, 544), codes=z(3, 272, dtype=F8), scales=z(3, 3, dtype=F32), gated=True)
    _refused(L, L.deer_quantize, good, dict(
        x=[z(3, 272), z(3, 544, dtype=F32)], codes=[z(3, 272), z(3, 544, dtype=F8)], scales=[z(3, 2, dtype=F32), z(3, 3)], gated=[False]))


def test_linear_operands(L):
    good = dict(x=z(3, 272, dtype=F8), x_scale=z(3, 3, dtype=F32), w=z(144, 272, dtype=F8), w_scale=z(2, 3, dtype=F32), y=z(3, 144), residual=z(3, 144))
    _refused(L, L.deer_linear_quant, good, dict(
        x=[z(3, 272), z(3, 256, dtype=F8)], x_scale=[z(3, 2, dtype=F32), z(3, 3)], w=[z(144, 272), z(144, 256, dtype=F8), z(160, 272, dtype=F8)],
        w_scale=[z(1, 3, dtype=F32), z(2, 2, dtype=F32), z(2, 3)], y=[z(3, 128), z(3, 144, dtype=F32)], residual=[z(1, 144), z(3, 144, dtype=F32)]))


def test_store_and_attention_operands(L):
    kv = L.KVCacheQuant.empty(8, 2, 64, 3, 4, device="cpu")
    rows, other = z(3, 5, 2, 64), z(3, 5, 4, 64)
    ids = z(3, dtype=I32)
    good = dict(kv=kv, seq_ids=ids, k_rows=rows, v_rows=rows, keep=ids)
    _refused(L, L.deer_kv_store, good, dict(
        seq_ids=[z(2, dtype=I32), z(3, dtype=torch.int64)], k_rows=[other, z(3, 5, 2, 128), z(3, 5, 2, 64, dtype=F32)],
        v_rows=[other, z(3, 4, 2, 64), z(3, 5, 2, 64, dtype=F32)], keep=[z(2, dtype=I32), z(3, dtype=torch.int64)]))
    need = L.deer_block_attn_quant_workspace_bytes(3, 5, 4, 2, 64, 48)
    good = dict(kv=kv, seq_ids=ids, q=z(3, 5, 4, 64), k_blk=rows, v_blk=rows, out=z(3, 5, 4, 64), row_state=z(3, 5, dtype=I32), mask=L.DEER_MASK_BIDIR,
                scale=0.125, max_seq_len=48, workspace=z(need + 16, dtype=torch.uint8))
    _refused(L, L.deer_block_attn_quant, good, dict(
        seq_ids=[z(2, dtype=I32), z(3, dtype=torch.int64)], q=[z(3, 5, 4, 128), z(3, 5, 4, 64, dtype=F32)], k_blk=[other, z(3, 4, 2, 64), rows.float()],
        v_blk=[other, z(3, 4, 2, 64), rows.float()], out=[z(3, 5, 2, 64), z(3, 5, 4, 64, dtype=F32)], row_state=[z(3, 4, dtype=I32), z(3, 5, dtype=torch.int64)]))


def test_a_bf16_cache_is_the_librarys_to_refuse(L):
    i32 = lambda *shape: z(*shape, dtype=I32)
    kv = L.KVCache(z(8, 2, 16, 64), z(8, 2, 16, 64), i32(3, 4), i32(3), i32(3), i32(8), i32(1))
    rows, ids = z(3, 5, 2, 64), i32(3)
    with pytest.raises(L.DeerError) as e:
        L.deer_kv_store(kv, ids, rows, rows, stream=1)
    assert e.value.code == L.DEER_ERR_UNSUPPORTED
    with pytest.raises(L.DeerError) as e:
        L.deer_block_attn_quant(kv, ids, z(3, 5, 4, 64), rows, rows, z(3, 5, 4, 64), None, L.DEER_MASK_CAUSAL, 0.125, 48, i32(1 << 16), stream=1)
    assert e.value.code == L.DEER_ERR_UNSUPPORTED

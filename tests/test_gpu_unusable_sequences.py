"""Sequences that a call cannot use are reported wherever they stand in it, in both kinds of cache."""
import math

import numpy as np
import pytest
import torch

from oracle import deer_oracle as O
from paper_2512_15176_b200 import workload as W
from tests.test_gpu_quant import _cache, check_attention

pytestmark = pytest.mark.gpu


def _call(lengths, ids, msl, bound, k=32, Hq=16, Hkv=2, D=128):
    from paper_2512_15176_b200 import binding as L
    kv, okv = _cache(lengths, Hkv, D, 0, 470)
    B = len(ids)
    q, kb, vb = (W.normal(470, n, (B, k, h, D), 1.0) for n, h in (("q", Hq), ("k", Hkv), ("v", Hkv)))
    out = torch.full((B, k, Hq, D), 5.0, dtype=torch.bfloat16, device="cuda")
    ws = torch.full((L.deer_block_attn_quant_workspace_bytes(B, k, Hq, Hkv, D, bound),), 255, dtype=torch.uint8, device="cuda")
    L.deer_block_attn_quant(kv, torch.tensor(ids, dtype=torch.int32, device="cuda"), q.cuda(), kb.cuda(), vb.cuda(), out, None, 0, 1 / math.sqrt(D), bound, ws)
    status = L.deer_kv_status(kv)
    return status, out, (q, kb, vb, okv)


@pytest.mark.parametrize("bound", [100, 1 << 20])
@pytest.mark.parametrize("ids", [[-1], [7, -1, 3], [9] * 33])
def test_no_usable_sequence_at_all_8_bit(ids, bound):
    from paper_2512_15176_b200 import binding as L
    status, out, _ = _call([40, 70], ids, 100, bound)
    assert status == L.DEER_ERR_INVALID_ARG and (out == 5).all()


@pytest.mark.parametrize("bound", [100, 1 << 20])
def test_unusable_sequences_behind_the_last_usable_one_8_bit(bound):
    from paper_2512_15176_b200 import binding as L
    lengths = [3 * s + 1 for s in range(32)]
    ids = list(range(32)) + [-1, 32, 99, -7, 40, 41, 42, 43]
    status, out, (q, kb, vb, okv) = _call(lengths, ids, 100, bound)
    assert status == L.DEER_ERR_INVALID_ARG and (out[32:] == 5).all()
    check_attention(out[:32], q[:32], kb[:32], vb[:32], okv, ids[:32], 0, 1 / math.sqrt(128), None, "usable")


def _call_bf16(lengths, ids, k=32, Hq=16, Hkv=2, D=128):
    from paper_2512_15176_b200 import binding as L
    cfg = W.StepConfig("unusable", len(lengths), Hq, Hkv, D, k, 64, 64, (1, 128), seed=471, growth=k)
    lay = W.kv_layout(cfg, np.asarray(lengths, dtype=np.int32))
    kp, vp = W.kv_pools(cfg, lay.num_pages, sigma=1.0)
    kv = L.KVCache.from_layout(lay, kp, vp)
    B, bound = len(ids), 128
    q, kb, vb = (W.normal(471, n, (B, k, h, D), 1.0) for n, h in (("q", Hq), ("k", Hkv), ("v", Hkv)))
    out = torch.full((B, k, Hq, D), 5.0, dtype=torch.bfloat16, device="cuda")
    ws = torch.full((L.deer_block_attn_workspace_bytes(B, k, Hq, Hkv, D, bound),), 255, dtype=torch.uint8, device="cuda")
    L.deer_block_attn(kv, torch.tensor(ids, dtype=torch.int32, device="cuda"), q.cuda(), kb.cuda(), vb.cuda(), out, 0, 0, 1 / math.sqrt(D), bound, ws)
    status = L.deer_kv_status(kv)
    want = lambda b: O.block_attention(q[b:b + 1].double().numpy(), kb[b:b + 1].double().numpy(), vb[b:b + 1].double().numpy(), kp.double().numpy(),
                                       vp.double().numpy(), lay.page_table, lay.seq_len, [ids[b]], 0, 1 / math.sqrt(D))
    return status, out, want


@pytest.mark.parametrize("ids", [[-1], [7, -1, 3], [9] * 33])
@pytest.mark.parametrize("D", [64, 128])
def test_no_usable_sequence_at_all_bf16(ids, D):
    from paper_2512_15176_b200 import binding as L
    status, out, _ = _call_bf16([40, 70], ids, D=D)
    assert status == L.DEER_ERR_INVALID_ARG and (out == 5).all()


def test_unusable_sequences_behind_the_last_usable_one_bf16():
    from paper_2512_15176_b200 import binding as L
    ids = list(range(32)) + [-1, 32, 99, -7, 40, 41, 42, 43]
    status, out, want = _call_bf16([3 * s + 1 for s in range(32)], ids)
    assert status == L.DEER_ERR_INVALID_ARG and (out[32:] == 5).all()
    for b in (0, 17, 31):
        w = want(b)
        # one bf16 rounding of the result, bf16 probabilities (2^-8 each) against values of order one
        assert np.abs(out[b:b + 1].double().cpu().numpy() - w).max() <= 2e-2

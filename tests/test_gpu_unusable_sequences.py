"""Sequences that a call cannot use are reported wherever they stand in it."""
import math

import pytest
import torch

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

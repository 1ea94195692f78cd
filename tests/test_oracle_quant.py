"""Pins of the oracle's 8-bit pieces: e4m3 rounding against torch's conversion, scales and codes against their
definition element by element, the store against a dense record of the tokens, and the attention over an 8-bit cache
against the bf16 definition on the values that the codes stand for."""
import math

import numpy as np
import pytest
import torch

from oracle import deer_oracle as O


def test_e4m3_round_is_the_conversion():
    codes = torch.arange(256, dtype=torch.int32).to(torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    vals = np.unique(codes[np.isfinite(codes)])
    assert vals.max() == 448 and len(vals) == 253
    np.testing.assert_array_equal(O.e4m3_round(vals), vals)
    mid = (vals[1:] + vals[:-1]) / 2                                       # halves: to the even code
    for v in (mid, mid * (1 + 1e-6), mid * (1 - 1e-6), np.linspace(-460, 460, 20011)):
        v = v.astype(np.float32)
        want = torch.from_numpy(np.clip(v, -448, 448)).to(torch.float8_e4m3fn).double().numpy()
        np.testing.assert_array_equal(O.e4m3_round(v), want)


@pytest.mark.parametrize("M,K", [(1, 16), (3, 128), (4, 208), (2, 640)])
def test_rows_follow_the_definition(M, K):
    rng = np.random.default_rng(5)
    y = rng.standard_normal((M, K))
    y[0] = 0.0
    codes, scales = O.quantise_rows(y)
    for m in range(M):
        for c in range(K):
            g = c // 128
            s = max(np.float32(np.abs(y[m, g * 128:(g + 1) * 128]).max()) / np.float32(448), np.float32(2.0 ** -126))
            assert scales[m, g] == s
            q = float(np.float32(y[m, c]) / s)
            assert abs(codes[m, c] - q) <= O.e4m3_step(q) / 2 + 1e-12
    back = O.dequantise_rows(codes, scales)
    err = np.abs(back - y)
    cap = np.repeat(scales.astype(np.float64), 128, axis=1)[:, :K]
    assert (err <= np.maximum(np.abs(y) * 2.0 ** -4, cap * 2.0 ** -10) * (1 + 1e-5)).all()


def test_weight_blocks():
    rng = np.random.default_rng(6)
    w = rng.standard_normal((144, 272)) * np.exp(rng.standard_normal((144, 1)))
    codes, scales = O.quantise_weight(w)
    assert scales.shape == (2, 3)
    assert scales[1, 2] == np.float32(np.abs(w[128:, 256:]).max()) / np.float32(448)
    assert np.abs(O.dequantise_weight(codes, scales) - w).max() <= np.abs(w).max() * 2.0 ** -4


def _bf16(rng, *shape):
    return torch.from_numpy(rng.standard_normal(shape)).to(torch.bfloat16).double().numpy()


@pytest.mark.parametrize("seed", [0, 1, 2])
def test_store_against_a_dense_record(seed):
    """Rounds of store + length update with random keeps: every token of a full page reads back as its page's
    quantisation (computed here from the record), every other exactly; rejected rows leave no trace."""
    rng = np.random.default_rng(seed)
    Hkv, D, S, pages = 2, 8, 2, 16
    table = rng.permutation(S * pages).reshape(S, pages)
    z = lambda *s: np.zeros(s)
    kv = O.QuantKV(z(S * pages, Hkv, 16, D), z(S * pages, Hkv, 16, D), z(S * pages, Hkv), z(S * pages, Hkv), z(S, Hkv, 48, D), z(S, Hkv, 48, D),
                   table, np.zeros(S, dtype=np.int64))
    record = [[np.zeros((0, Hkv, D)), np.zeros((0, Hkv, D))] for _ in range(S)]
    for _ in range(9):
        k = int(rng.integers(1, 33))
        kr, vr = _bf16(rng, S, k, Hkv, D), _bf16(rng, S, k, Hkv, D)
        keep = rng.integers(0, k + 1, size=S)
        kv.store(np.arange(S), kr, vr, keep)
        for s in range(S):
            for x, rows in ((0, kr), (1, vr)):
                record[s][x] = np.concatenate([record[s][x], rows[s, :keep[s]]])
        kv.seq_len = kv.seq_len + keep
        for s in range(S):
            n = len(record[s][0])
            assert kv.seq_len[s] == n
            for x, got in enumerate(kv.gather(s)):
                want = record[s][x].copy()
                for p in range(n // 16):
                    for h in range(Hkv):
                        part = record[s][x][p * 16:(p + 1) * 16, h]
                        sc = np.float32(np.abs(part).max()) / np.float32(448)
                        q = torch.from_numpy(part.astype(np.float32) / sc).to(torch.float8_e4m3fn).double().numpy()
                        want[p * 16:(p + 1) * 16, h] = q * float(sc)
                np.testing.assert_array_equal(got, want)


def test_attention_is_the_definition_on_the_dequantised_tokens():
    rng = np.random.default_rng(9)
    B, k, Hq, Hkv, D, P = 2, 5, 4, 2, 16, 4
    table = rng.permutation(B * P).reshape(B, P)
    codes = lambda: O.e4m3_round(rng.standard_normal((B * P, Hkv, 16, D)) * 50)
    kv = O.QuantKV(codes(), codes(), rng.random((B * P, Hkv)) / 50, rng.random((B * P, Hkv)), rng.standard_normal((B, Hkv, 48, D)),
                   rng.standard_normal((B, Hkv, 48, D)), table, np.array([37, 16]))
    q, kb, vb = (rng.standard_normal((B, k, h, D)) for h in (Hq, Hkv, Hkv))
    out = O.quant_block_attention(q, kb, vb, kv, np.arange(B), O.MASK_CAUSAL, 1 / math.sqrt(D))
    for b, n in enumerate((37, 16)):
        for i in range(k):
            for h in range(Hq):
                g = h // 2
                ks, vs = [], []
                for t in range(n + i + 1):
                    if t >= n:
                        ks.append(kb[b, t - n, g]); vs.append(vb[b, t - n, g])
                    elif t < n // 16 * 16:
                        pg = table[b, t // 16]
                        ks.append(kv.codes[0][pg, g, t % 16] * float(kv.scale[0][pg, g])); vs.append(kv.codes[1][pg, g, t % 16] * float(kv.scale[1][pg, g]))
                    else:
                        ks.append(kv.tail[0][b, g, t % 48]); vs.append(kv.tail[1][b, g, t % 48])
                z = np.array([np.dot(q[b, i, h], x) for x in ks]) / math.sqrt(D)
                w = np.exp(z - z.max())
                np.testing.assert_allclose(out[b, i, h], sum(a * v for a, v in zip(w / w.sum(), vs)), rtol=1e-10, atol=1e-12)

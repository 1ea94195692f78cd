"""The 8-bit calls on the GPU against the oracle in 64 bits.

Tolerances, derived:
  codes      the device's quotient y / s may differ from the oracle's by the fp32 roundings on the way (DELTA, relative), so a
             code is within half an e4m3 step of the oracle's quotient plus that; s within 2 DELTA.
  linear     one bf16 rounding of the result (2^-8), and fp32 accumulation: at most (K / 128 + 16) additions of 2^-24
             relative to the sum of magnitudes for K <= 16384, i.e. below 2^-16 of it.
  attention  one bf16 rounding (2^-8), and probabilities with 9 significant bits or more (2^-9 each, of sum p |v|);
             the scores' fp32 sums move p by less than 2^-12 at these magnitudes.
"""
import math

import numpy as np
import pytest
import torch

from oracle import deer_oracle as O
from paper_2512_15176_b200 import workload as W

pytestmark = pytest.mark.gpu

F8 = torch.float8_e4m3fn


def f64(t):
    return t.to(torch.float64).cpu().numpy()


def check_codes(codes, scales, y64, delta, label):
    """codes [M, K], scales [M, G] of the device against the fp64 values y64."""
    K = y64.shape[1]
    got, s = f64(codes), f64(scales)
    G = -(-K // 128)
    want_s = np.stack([np.maximum(np.abs(y64[:, g * 128:(g + 1) * 128]).max(axis=1) / 448.0, 2.0 ** -126) for g in range(G)], 1)
    assert (np.abs(s - want_s) <= 2 * delta * want_s).all(), label
    q = y64 / np.repeat(want_s, 128, axis=1)[:, :K]
    err = np.abs(got - np.clip(q, -448, 448))
    tol = O.e4m3_step(q) / 2 + 4 * delta * np.abs(q) + 1e-12
    assert np.isfinite(got).all() and (err <= tol).all(), f"{label}: {np.max(err - tol)}"


@pytest.mark.parametrize("M,K,res,total", [(1, 16, False, False), (3, 128, True, True), (37, 2048, True, True), (5, 2064, True, False),
                                           (2, 4096, False, True), (9, 4112, True, True), (4, 8192, True, True), (3, 8208, False, False),
                                           (2, 16400, True, True), (1, 65536, True, True), (300, 144, True, True)])
def test_rmsnorm_quant(M, K, res, total):
    from paper_2512_15176_b200 import binding as L
    x, g = W.normal(201, "x", (M, K), 1.7), W.normal(201, "g", (K,), 1.0)
    r = W.normal(201, "r", (M, K), 1.0) if res else None
    x[0, :: 41] *= 30.0
    G = -(-K // 128)
    codes = torch.full((M + 1, K), 2.0, device="cuda").to(F8)
    scales = torch.full((M + 1, G), 7.0, device="cuda")
    tot = torch.full((M + 1, K), 5.0, dtype=torch.bfloat16, device="cuda")
    L.deer_rmsnorm_quant(x.cuda(), g.cuda(), codes[:M], scales[:M], 1e-6, residual=r.cuda() if res else None, total=tot[:M] if total else None)
    torch.cuda.synchronize()
    h = f64(x) + (f64(r) if res else 0.0)
    check_codes(codes[:M], scales[:M], O.rmsnorm(h, f64(g), 1e-6), 2e-6, f"rmsnorm {M}x{K}")
    if total:
        assert (f64(tot[:M]) == f64(torch.from_numpy(h.astype(np.float32)).to(torch.bfloat16))).all()
    # what lies behind the last row stays
    assert (f64(codes[M]) == 2).all() and (scales[M] == 7).all() and (tot[M] == 5).all()


def test_rmsnorm_quant_total_in_place():
    from paper_2512_15176_b200 import binding as L
    M, K = 33, 4096
    x, r, g = (W.normal(202, n, s, 1.0).cuda() for n, s in (("x", (M, K)), ("r", (M, K)), ("g", (K,))))
    outs = []
    for into in (None, "x", "r"):
        xx, rr = x.clone(), r.clone()
        tot = {None: torch.empty_like(x), "x": xx, "r": rr}[into]
        codes, scales = torch.empty(M, K, dtype=F8, device="cuda"), torch.empty(M, 32, device="cuda")
        L.deer_rmsnorm_quant(xx, g, codes, scales, 1e-6, residual=rr, total=tot)
        outs.append((codes.view(torch.uint8), scales, tot))
    for o in outs[1:]:
        assert all(torch.equal(a, b) for a, b in zip(outs[0], o))


@pytest.mark.parametrize("M,K,gated", [(1, 16, False), (3, 128, True), (33, 208, True), (5, 4096, False), (64, 1536, True), (257, 1040, False)])
def test_quantize(M, K, gated):
    from paper_2512_15176_b200 import binding as L
    x = W.normal(203, "x", (M, 2 * K if gated else K), 2.0)
    G = -(-K // 128)
    codes = torch.full((M + 1, K), 2.0, device="cuda").to(F8)
    scales = torch.full((M + 1, G), 7.0, device="cuda")
    L.deer_quantize(x.cuda(), codes[:M], scales[:M], gated=gated)
    torch.cuda.synchronize()
    x64 = f64(x)
    y = O.swiglu(x64[:, :K], x64[:, K:]) if gated else x64
    if gated:
        check_codes(codes[:M], scales[:M], y, 8e-6, f"gated {M}x{K}")
    else:                                                  # nothing is rounded before the quotient: bit-exact
        want_c, want_s = O.quantise_rows(y)
        assert (f64(codes[:M]) == want_c).all() and (scales[:M].cpu().numpy() == want_s).all()
    assert (f64(codes[M]) == 2).all() and (scales[M] == 7).all()


def test_quantize_zeros_nan_inf_and_tiny_groups():
    """A group of zeros has codes 0; a NaN or an infinity poisons its own group of 128 columns and no other."""
    from paper_2512_15176_b200 import binding as L
    x = W.normal(204, "x", (4, 512), 1.0)
    x[0] = 0.0
    x[1, 130] = float("nan")
    x[2, 300] = float("inf")
    x[3, :128] = 2.0 ** -130                               # subnormal: below the smallest scale
    codes, scales = torch.empty(4, 512, dtype=F8, device="cuda"), torch.empty(4, 4, device="cuda")
    L.deer_quantize(x.cuda(), codes, scales)
    v = (codes.float().view(4, 4, 128) * scales[:, :, None]).cpu()
    assert (v[0] == 0).all() and (scales[0] == 2.0 ** -126).all()
    assert v[1, 1].isnan().all() and v[1, [0, 2, 3]].isfinite().all()
    assert v[2, 2].isnan().all() and v[2, [0, 1, 3]].isfinite().all()
    assert (v[3, 0] == 2.0 ** -130).all()


def _linear_inputs(M, K, N, seed=205):
    x, w = W.normal(seed, "x", (M, K), 1.0, dtype=torch.float32), W.normal(seed, "w", (N, K), 1.0, dtype=torch.float32)
    w = w * torch.exp(torch.linspace(-2, 2, N))[:, None]
    xc, xs = O.quantise_rows(f64(x))
    wc, ws = O.quantise_weight(f64(w))
    dev = lambda c: torch.from_numpy(c).float().to(F8).cuda()
    return (dev(xc), torch.from_numpy(xs).cuda(), dev(wc), torch.from_numpy(ws).cuda()), O.dequantise_rows(xc, xs), O.dequantise_weight(wc, ws)


@pytest.mark.parametrize("M,K,N,res", [(1, 128, 128, False), (1, 4096, 4096, True), (7, 1024, 272, True), (16, 16, 16, False), (17, 208, 144, True),
                                       (32, 4096, 1024, True), (33, 640, 2000, False), (64, 2048, 512, True), (65, 1296, 400, True),
                                       (128, 1024, 1040, True), (129, 512, 4096, False), (256, 2048, 384, True), (300, 1536, 656, True),
                                       (513, 272, 128, True), (32, 12288, 256, False)])
def test_linear_quant(M, K, N, res):
    from paper_2512_15176_b200 import binding as L
    dev, x64, w64 = _linear_inputs(M, K, N)
    r = W.normal(205, "r", (M, N), 3.0) if res else None
    y = torch.full((M + 1, N), 9.0, dtype=torch.bfloat16, device="cuda")
    L.deer_linear_quant(*dev, y[:M], residual=r.cuda() if res else None)
    torch.cuda.synchronize()
    want = x64 @ w64.T + (f64(r) if res else 0.0)
    tol = 2.0 ** -8 * np.abs(want) + 2.0 ** -16 * (np.abs(x64) @ np.abs(w64).T) + 1e-30
    err = np.abs(f64(y[:M]) - want)
    assert np.isfinite(f64(y[:M])).all() and (err <= tol).all(), f"{np.max(err / tol)}"
    assert (y[M] == 9).all()
    # the same bits again, and with the residual in place of the output
    y2 = r.cuda() if res else torch.empty_like(y[:M])
    L.deer_linear_quant(*dev, y2, residual=y2 if res else None)
    assert torch.equal(y2, y[:M])


def test_linear_quant_nan_stays_in_its_row_and_column():
    from paper_2512_15176_b200 import binding as L
    (x, xs, w, ws), _, _ = _linear_inputs(40, 512, 384)
    xs[5, 2] = float("nan")
    ws[1, 3] = float("inf")                                # rows 128 .. 255 of w
    y = torch.empty(40, 384, dtype=torch.bfloat16, device="cuda")
    L.deer_linear_quant(x, xs, w, ws, y)
    bad = ~y.isfinite()
    assert bad[5].all() and bad[:, 128:256].all()
    bad[5] = False
    bad[:, 128:256] = False
    assert not bad.any()


# ---- the 8-bit cache -------------------------------------------------------------------------------------------

def _cache(lengths, Hkv, D, room, seed, spare=3, device="cuda"):
    """A cache with random codes, scales and tails on the device, and the oracle's copy of it.  Pages in random order;
    every sequence can hold its length plus `room`."""
    from paper_2512_15176_b200 import binding as L
    rng = np.random.default_rng(seed)
    need = [-(-(n + room) // 16) for n in lengths]
    total, width, S = sum(need) + spare, max(max(need), 1), len(lengths)
    order = rng.permutation(total)
    table = np.full((S, width), -1, dtype=np.int32)
    at = 0
    for s, c in enumerate(need):
        table[s, :c] = order[at:at + c]
        at += c
    free = order[at:]
    stack = np.zeros(total, dtype=np.int32)
    stack[:len(free)] = free
    g = torch.Generator().manual_seed(seed)
    codes = lambda: (torch.randn(total, Hkv, 16, D, generator=g) * 120).clamp(-448, 448).to(F8)
    scale = lambda: torch.exp(torch.randn(total, Hkv, generator=g)) / 120
    tail = lambda: torch.randn(S, Hkv, 48, D, generator=g).to(torch.bfloat16)
    kp, vp, ks, vs, kt, vt = codes(), codes(), scale(), scale(), tail(), tail()
    i32 = lambda a: torch.as_tensor(np.asarray(a, dtype=np.int32), device=device)
    kv = L.KVCacheQuant(*(t.to(device) for t in (kp, vp, ks, vs, kt, vt)), i32(table), i32(lengths), i32(need), i32(stack), i32([len(free)]))
    okv = O.QuantKV(f64(kp), f64(vp), ks.numpy(), vs.numpy(), f64(kt), f64(vt), table, np.asarray(lengths))
    return kv, okv


def _same_cache(kv, okv, label=""):
    for x, (pool, scale, tail) in enumerate(((kv.k_pool, kv.k_scale, kv.k_tail), (kv.v_pool, kv.v_scale, kv.v_tail))):
        assert (scale.cpu().numpy() == okv.scale[x]).all(), label
        assert (f64(pool) == okv.codes[x]).all(), label
        assert (f64(tail) == okv.tail[x]).all(), label


def _ids(n):
    return torch.arange(n, dtype=torch.int32, device="cuda")


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("lengths,k,keep", [([0], 1, [1]), ([15], 1, [1]), ([15, 16, 17, 0], 1, [1, 1, 0, 1]), ([3, 31, 47, 100], 32, [32, 17, 1, 0]),
                                            ([14, 30], 18, [18, 2]), ([0, 5, 16], 77, [77, 60, 76]), ([9, 1], 400, [399, 64]), ([40], 5, [3])])
def test_store(lengths, k, keep, D):
    """Bit-exact pools, scales and tails, what the call does not touch included; repeated, it changes nothing."""
    from paper_2512_15176_b200 import binding as L
    kv, okv = _cache(lengths, 2, D, k, 301)
    B = len(lengths)
    kr, vr = W.normal(301, "k", (B, k, 2, D), 1.0), W.normal(301, "v", (B, k, 2, D), 3.0)
    kr[0, 0] = 0.0
    ids = list(range(B))[::-1]
    dev = [torch.tensor(ids, dtype=torch.int32, device="cuda"), kr.cuda(), vr.cuda(), torch.tensor(keep, dtype=torch.int32, device="cuda")]
    okv.store(ids, f64(kr), f64(vr), keep)
    for turn in range(2 if k <= 32 else 1):
        L.deer_kv_store(kv, *dev)
        torch.cuda.synchronize()
        assert L.deer_kv_status(kv) == 0
        _same_cache(kv, okv, f"turn {turn}")
    assert (kv.seq_len.cpu().numpy() == okv.seq_len).all()


def test_store_clamps_keep_and_reports_unmapped_pages():
    from paper_2512_15176_b200 import binding as L
    kv, okv = _cache([10, 20], 2, 64, 32, 302)
    kr, vr = W.normal(302, "k", (2, 8, 2, 64), 1.0), W.normal(302, "v", (2, 8, 2, 64), 1.0)
    L.deer_kv_store(kv, _ids(2), kr.cuda(), vr.cuda(), torch.tensor([99, -5], dtype=torch.int32, device="cuda"))
    okv.store([0, 1], f64(kr), f64(vr), [8, 0])
    _same_cache(kv, okv)
    kv.page_table[0, 0] = -1
    before = kv.k_pool.view(torch.uint8).clone()
    L.deer_kv_store(kv, _ids(1), kr[:1].cuda(), vr[:1].cuda())
    assert L.deer_kv_status(kv) == L.DEER_ERR_BAD_PAGE and torch.equal(before, kv.k_pool.view(torch.uint8))
    kv.page_table[0, 0] = kv.k_pool.shape[0]
    L.deer_kv_store(kv, _ids(1), kr[:1].cuda(), vr[:1].cuda())
    assert L.deer_kv_status(kv) == L.DEER_ERR_BAD_PAGE and torch.equal(before, kv.k_pool.view(torch.uint8))
    L.deer_kv_store(kv, _ids(1) + 7, kr[:1].cuda(), vr[:1].cuda())
    assert L.deer_kv_status(kv) == L.DEER_ERR_INVALID_ARG


def check_attention(out, q, kb, vb, okv, ids, mask, scale, states, label):
    q64, k64, v64 = f64(q), f64(kb), f64(vb)
    want = O.quant_block_attention(q64, k64, v64, okv, ids, mask, scale, states)
    a = O.QuantKV(okv.codes[0], np.abs(okv.codes[1]), *okv.scale, okv.tail[0], np.abs(okv.tail[1]), okv.page_table, okv.seq_len)
    mass = O.quant_block_attention(q64, k64, np.abs(v64), a, ids, mask, scale, states)       # sum p |v|
    got = f64(out)
    err, tol = np.abs(got - want), 2.0 ** -8 * np.abs(want) + (2.0 ** -9 + 2.0 ** -12) * mass + 1e-30
    assert np.isfinite(got).all(), label
    assert (err <= tol).all(), f"{label}: {np.max(err / tol)}"


CASES = [
    # lengths, k, Hq, Hkv, D, mask
    ([0], 1, 2, 1, 64, "causal"), ([1], 1, 8, 8, 128, "causal"), ([15, 16, 17], 1, 4, 2, 128, "causal"), ([0, 31, 33], 5, 8, 2, 64, "causal"),
    ([1003], 1, 32, 8, 128, "causal"), ([5000, 3], 1, 8, 2, 64, "causal"), ([300, 77, 1024], 32, 16, 4, 128, "causal"),
    ([129, 0], 32, 8, 1, 128, "bidir"), ([700, 16], 17, 6, 2, 128, "states"), ([31, 250, 0, 64], 32, 4, 4, 64, "states"),
    ([2500], 32, 32, 8, 128, "causal"), ([1500, 1111], 32, 16, 2, 128, "states"), ([640], 31, 7, 1, 128, "causal"), ([97], 9, 40, 2, 128, "bidir"),
]


@pytest.mark.parametrize("lengths,k,Hq,Hkv,D,mask", CASES)
def test_attention(lengths, k, Hq, Hkv, D, mask):
    from paper_2512_15176_b200 import binding as L
    B = len(lengths)
    kv, okv = _cache(lengths, Hkv, D, 0, 401)
    q, kb, vb = (W.normal(401, n, (B, k, h, D), 1.0) for n, h in (("q", Hq), ("k", Hkv), ("v", Hkv)))
    states = None
    if mask == "states":
        states = W.rng(401, "states").integers(-1, 2, size=(B, k)).astype(np.int32)
        states[-1] = -1                                    # a sequence whose rows are all absent
    m = L.DEER_MASK_CAUSAL if mask == "causal" else L.DEER_MASK_BIDIR
    ids = list(range(B))[::-1]
    out = torch.full((B + 1, k, Hq, D), float("nan"), dtype=torch.bfloat16, device="cuda")
    msl = max(lengths)
    need = L.deer_block_attn_quant_workspace_bytes(B, k, Hq, Hkv, D, msl)
    ws = torch.full((need + 64,), 255, dtype=torch.uint8, device="cuda")          # NaN patterns: nothing unwritten may be read
    L.deer_block_attn_quant(kv, torch.tensor(ids, dtype=torch.int32, device="cuda"), q.cuda(), kb.cuda(), vb.cuda(), out[:B],
                            None if states is None else torch.from_numpy(states).cuda(), m, 1 / math.sqrt(D), msl, ws[:need])
    torch.cuda.synchronize()
    assert L.deer_kv_status(kv) == 0
    check_attention(out[:B], q, kb, vb, okv, ids, m, 1 / math.sqrt(D), states, f"{lengths} {k} {mask}")
    assert out[B].isnan().all() and (ws[need:] == 255).all()


@pytest.mark.parametrize("B,k,Hq,Hkv,hi,mask", [(24, 9, 16, 8, 70, "causal"), (40, 32, 8, 2, 300, "states"), (900, 5, 32, 8, 20, "causal"),
                                                (12, 32, 32, 4, 900, "bidir")])
def test_attention_many_short_sequences(B, k, Hq, Hkv, hi, mask):
    """More (sequence, KV head) units than thread blocks: a block walks many of them, most with one to a few tiles, in
    lists of at most 48; two calls in a row (a block's hand-overs between units may not depend on timing)."""
    from paper_2512_15176_b200 import binding as L
    rng = np.random.default_rng(410)
    lengths = [int(x) for x in rng.integers(0, hi + 1, size=B)]
    D = 128
    kv, okv = _cache(lengths, Hkv, D, 0, 410)
    q, kb, vb = (W.normal(410, n, (B, k, h, D), 1.0) for n, h in (("q", Hq), ("k", Hkv), ("v", Hkv)))
    states = rng.integers(-1, 2, size=(B, k)).astype(np.int32) if mask == "states" else None
    m = L.DEER_MASK_CAUSAL if mask == "causal" else L.DEER_MASK_BIDIR
    ws = torch.full((L.deer_block_attn_quant_workspace_bytes(B, k, Hq, Hkv, D, hi),), 255, dtype=torch.uint8, device="cuda")
    outs = [torch.full((B, k, Hq, D), float("nan"), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    dev = [t.cuda() for t in (q, kb, vb)]
    for out in outs:
        L.deer_block_attn_quant(kv, _ids(B), *dev, out, None if states is None else torch.from_numpy(states).cuda(), m, 1 / math.sqrt(D), hi, ws)
    assert L.deer_kv_status(kv) == 0
    assert torch.equal(outs[0], outs[1])
    check_attention(outs[0], q, kb, vb, okv, list(range(B)), m, 1 / math.sqrt(D), states, f"{B} {k} {mask}")


@pytest.mark.parametrize("k,Hq,Hkv,D", [(1, 4, 1, 128), (8, 4, 2, 64), (32, 16, 4, 128), (16, 8, 1, 128)])
def test_attention_spread_scales_and_scores(k, Hq, Hkv, D):
    """Page scales over forty octaves (pages of zeros among them), a dominating key late in the context over a long
    background whose tiny weights add up, and queries of very different size."""
    from paper_2512_15176_b200 import binding as L
    n = 2000
    kv, okv = _cache([n], Hkv, D, 0, 402)
    rng = np.random.default_rng(402)
    vs = np.exp2(rng.uniform(-20, 20, size=okv.scale[1].shape)).astype(np.float32)
    vs[rng.integers(0, len(vs), 9)] = np.float32(2.0 ** -126)
    okv.scale[1][:] = vs
    zero = int(okv.page_table[0, 5])
    okv.codes[1][zero] = 0.0
    okv.codes[0][int(okv.page_table[0, 7])] = 0.0
    okv.scale[0][:] = (okv.scale[0] * 0.02).astype(np.float32)                 # a flat background ...
    big = int(okv.page_table[0, 100])
    okv.scale[0][big] = np.float32(0.02)
    kv.v_scale.copy_(torch.from_numpy(okv.scale[1]))
    kv.k_scale.copy_(torch.from_numpy(okv.scale[0]))
    kv.v_pool.copy_(torch.from_numpy(okv.codes[1]).float().to(F8))
    kv.k_pool.copy_(torch.from_numpy(okv.codes[0]).float().to(F8))
    q, kb, vb = (W.normal(402, x, (1, k, h, D), 1.0) for x, h in (("q", Hq), ("k", Hkv), ("v", Hkv)))
    q[0, 0] *= 2.0 ** -20
    if k > 2:
        q[0, 1] = 0.0
    out = torch.empty(1, k, Hq, D, dtype=torch.bfloat16, device="cuda")
    ws = torch.full((L.deer_block_attn_quant_workspace_bytes(1, k, Hq, Hkv, D, n),), 255, dtype=torch.uint8, device="cuda")
    L.deer_block_attn_quant(kv, _ids(1), q.cuda(), kb.cuda(), vb.cuda(), out, None, L.DEER_MASK_CAUSAL, 1 / math.sqrt(D), n, ws)
    check_attention(out, q, kb, vb, okv, [0], 0, 1 / math.sqrt(D), None, "spread")


@pytest.mark.parametrize("k,Hq,Hkv,D", [(4, 2, 1, 64), (32, 16, 4, 128), (20, 8, 1, 128)])
@pytest.mark.parametrize("what", ["nan", "inf"])
def test_attention_nonfinite_rows_reach_only_rows_that_see_them(k, Hq, Hkv, D, what):
    from paper_2512_15176_b200 import binding as L
    n, bad = 200, float(what)
    kv, okv = _cache([n], Hkv, D, 0, 403)
    q, kb, vb = (W.normal(403, x, (1, k, h, D), 1.0) for x, h in (("q", Hq), ("k", Hkv), ("v", Hkv)))
    clean = (q.clone(), kb.clone(), vb.clone())
    j = k - 2
    vb[0, j, 0, 3] = bad                                   # seen by rows j.. (causal)
    kb[0, k - 1, 0, 5] = float("nan")                      # seen by the last row alone
    ws = torch.empty(L.deer_block_attn_quant_workspace_bytes(1, k, Hq, Hkv, D, n), dtype=torch.uint8, device="cuda")
    out = torch.empty(1, k, Hq, D, dtype=torch.bfloat16, device="cuda")
    run = lambda m, st: L.deer_block_attn_quant(kv, _ids(1), q.cuda(), kb.cuda(), vb.cuda(), out, st, m, 1 / math.sqrt(D), n, ws)
    run(L.DEER_MASK_CAUSAL, None)
    G = Hq // Hkv
    got = out.float().cpu()
    assert got[0, :j].isfinite().all()
    assert (got[0, j, :G, 3].isnan() if what == "nan" else got[0, j, :G, 3] == bad).all()
    assert got[0, j, :G, :3].isfinite().all() and got[0, j, :G, 4:].isfinite().all()
    assert got[0, k - 1, :G].isnan().all()
    assert got[0, :, G:].isfinite().all()                  # the other KV heads' rows
    want = O.quant_block_attention(f64(clean[0]), f64(clean[1]), f64(clean[2]), okv, [0], 0, 1 / math.sqrt(D))
    assert np.abs(f64(out[0, :j]) - want[0, :j]).max() <= 2.0 ** -6 * np.abs(want).max()
    # absent positions hold anything
    st = torch.zeros(1, k, dtype=torch.int32)
    st[0, j:] = -1
    st[0, 0] = 1
    run(L.DEER_MASK_BIDIR, st.cuda())
    check_attention(out, clean[0], torch.where(kb.isfinite(), kb, 0), torch.where(vb.isfinite(), vb, 0), okv, [0], 1, 1 / math.sqrt(D), st.numpy(), "absent")


def test_attention_skips_sequences_it_cannot_use():
    from paper_2512_15176_b200 import binding as L
    kv, okv = _cache([40, 500], 2, 128, 0, 404)
    q, kb, vb = (W.normal(404, x, (2, 4, h, 128), 1.0).cuda() for x, h in (("q", 4), ("k", 2), ("v", 2)))
    out = torch.full((2, 4, 4, 128), 3.0, dtype=torch.bfloat16, device="cuda")
    ws = torch.empty(L.deer_block_attn_quant_workspace_bytes(2, 4, 4, 2, 128, 100), dtype=torch.uint8, device="cuda")
    L.deer_block_attn_quant(kv, _ids(2), q, kb, vb, out, None, 0, 0.1, 100, ws)           # sequence 1 is longer than max_seq_len
    assert L.deer_kv_status(kv) == L.DEER_ERR_INVALID_ARG
    check_attention(out[:1], q[:1], kb[:1], vb[:1], okv, [0], 0, 0.1, None, "first")
    kv.page_table[0, 1] = kv.k_pool.shape[0] + 5
    L.deer_block_attn_quant(kv, _ids(1), q[:1], kb[:1], vb[:1], out[:1], None, 0, 0.1, 100, ws)
    assert L.deer_kv_status(kv) == L.DEER_ERR_BAD_PAGE


@pytest.mark.parametrize("k", [1, 32])
def test_pools_past_four_gigabytes(k):
    """Pages at the far end of pools of more than 2^32 bytes: store there, then read."""
    from paper_2512_15176_b200 import binding as L
    Hkv, D, pages = 8, 128, (1 << 32) // (8 * 16 * 128) + 40
    kv = L.KVCacheQuant.empty(pages, Hkv, D, 1, 8)
    kv.free_stack.copy_(torch.arange(pages, dtype=torch.int32, device="cuda"))            # the highest pages first
    kr, vr = W.normal(405, "k", (1, 100, Hkv, D), 1.0), W.normal(405, "v", (1, 100, Hkv, D), 1.0)
    L.deer_kv_reserve_rows(kv, _ids(1), 100)
    L.deer_kv_store(kv, _ids(1), kr.cuda(), vr.cuda())
    L.deer_kv_commit_rows(kv, _ids(1), torch.tensor([100], dtype=torch.int32, device="cuda"), 100)
    assert L.deer_kv_status(kv) == 0
    table = kv.page_table.cpu().numpy()
    assert table[0, 0] == pages - 1 and kv.seq_len.item() == 100
    z = lambda *s: np.zeros(s)
    okv = O.QuantKV(z(7, Hkv, 16, D), z(7, Hkv, 16, D), z(7, Hkv), z(7, Hkv), z(1, Hkv, 48, D), z(1, Hkv, 48, D), np.arange(7)[None], np.array([0]))
    okv.store([0], f64(kr), f64(vr), [100])
    okv.seq_len[:] = 100
    assert (f64(kv.k_pool[torch.from_numpy(table[0, :6].astype(np.int64)).cuda()].float()) == okv.codes[0][:6]).all()
    q, kb, vb = (W.normal(406, x, (1, k, h, D), 1.0) for x, h in (("q", 32), ("k", Hkv), ("v", Hkv)))
    out = torch.empty(1, k, 32, D, dtype=torch.bfloat16, device="cuda")
    ws = torch.empty(L.deer_block_attn_quant_workspace_bytes(1, k, 32, Hkv, D, 100), dtype=torch.uint8, device="cuda")
    L.deer_block_attn_quant(kv, _ids(1), q.cuda(), kb.cuda(), vb.cuda(), out, None, 0, 1 / math.sqrt(D), 100, ws)
    check_attention(out, q, kb, vb, okv, [0], 0, 1 / math.sqrt(D), None, "far pages")


def test_reserve_store_commit_soak():
    """Rounds of reserve, attention, store and commit with random keeps, rejected rows included, then a prompt: the
    cache and the lengths follow the oracle bit by bit, the attention within its tolerance."""
    from paper_2512_15176_b200 import binding as L
    Hkv, Hq, D, S = 2, 8, 128, 3
    kv = L.KVCacheQuant.empty(64, Hkv, D, S, 24)
    z = lambda *s: np.zeros(s)
    okv = O.QuantKV(z(64, Hkv, 16, D), z(64, Hkv, 16, D), z(64, Hkv), z(64, Hkv), z(S, Hkv, 48, D), z(S, Hkv, 48, D), np.zeros((S, 24), dtype=np.int64),
                    np.zeros(S, dtype=np.int64))
    rng = np.random.default_rng(7)
    for turn in range(8):
        k = 90 if turn == 0 else int(rng.integers(1, 33))
        kr, vr = W.normal(500 + turn, "k", (S, k, Hkv, D), 1.0), W.normal(500 + turn, "v", (S, k, Hkv, D), 1.0)
        keep = rng.integers(0, k + 1, size=S)
        kd = torch.tensor(keep, dtype=torch.int32, device="cuda")
        (L.deer_kv_reserve_rows if k > 32 else L.deer_kv_reserve)(kv, _ids(S), k)
        okv.page_table = kv.page_table.cpu().numpy()
        if k <= 32:
            q = W.normal(500 + turn, "q", (S, k, Hq, D), 1.0)
            out = torch.empty(S, k, Hq, D, dtype=torch.bfloat16, device="cuda")
            msl = int(okv.seq_len.max())
            ws = torch.empty(L.deer_block_attn_quant_workspace_bytes(S, k, Hq, Hkv, D, msl), dtype=torch.uint8, device="cuda")
            L.deer_block_attn_quant(kv, _ids(S), q.cuda(), kr.cuda(), vr.cuda(), out, None, 0, 1 / math.sqrt(D), msl, ws)
            check_attention(out, q, kr, vr, okv, np.arange(S), 0, 1 / math.sqrt(D), None, f"turn {turn}")
        L.deer_kv_store(kv, _ids(S), kr.cuda(), vr.cuda(), kd)
        okv.store(np.arange(S), f64(kr), f64(vr), keep)
        (L.deer_kv_commit_rows if k > 32 else L.deer_kv_commit)(kv, _ids(S), kd, k)
        okv.seq_len = okv.seq_len + keep
        assert L.deer_kv_status(kv) == 0
        assert (kv.seq_len.cpu().numpy() == okv.seq_len).all()
        assert (kv.n_pages.cpu().numpy() == -(-okv.seq_len // 16)).all()
        _same_cache(kv, okv, f"turn {turn}")


@pytest.fixture()
def long_bound(monkeypatch):
    """The attention called with a bound on the lengths that is far above them: the kernel for long contexts, whatever the
    lengths are (short calls take another one)."""
    from paper_2512_15176_b200 import binding as L
    real = L.deer_block_attn_quant

    def call(kv, ids, q, kb, vb, out, states, mask, scale, msl, ws):
        B, k, Hq, D = q.shape
        ws = torch.full((L.deer_block_attn_quant_workspace_bytes(B, k, Hq, kv.n_kv_heads, D, 1 << 20),), 255, dtype=torch.uint8, device="cuda")
        real(kv, ids, q, kb, vb, out, states, mask, scale, 1 << 20, ws)

    monkeypatch.setattr(L, "deer_block_attn_quant", call)


@pytest.mark.parametrize("lengths,k,Hq,Hkv,D,mask", CASES)
def test_attention_under_a_long_bound(long_bound, lengths, k, Hq, Hkv, D, mask):
    test_attention(lengths, k, Hq, Hkv, D, mask)


@pytest.mark.parametrize("k,Hq,Hkv,D", [(32, 16, 4, 128), (16, 8, 1, 128), (5, 16, 2, 128)])
def test_spread_scales_under_a_long_bound(long_bound, k, Hq, Hkv, D):
    test_attention_spread_scales_and_scores(k, Hq, Hkv, D)


@pytest.mark.parametrize("k,Hq,Hkv,D", [(32, 16, 4, 128), (20, 8, 1, 128)])
@pytest.mark.parametrize("what", ["nan", "inf"])
def test_nonfinite_rows_under_a_long_bound(long_bound, k, Hq, Hkv, D, what):
    test_attention_nonfinite_rows_reach_only_rows_that_see_them(k, Hq, Hkv, D, what)


@pytest.mark.parametrize("scale", [0.0, -0.05])
@pytest.mark.parametrize("n,msl", [(100, 100), (3000, 1 << 20)])
def test_attention_with_a_scale_that_is_not_positive(n, msl, scale):
    """Zero: every visible key weighs the same; below zero: the least similar key weighs most."""
    from paper_2512_15176_b200 import binding as L
    k, Hq, Hkv, D = 32, 16, 4, 128
    kv, okv = _cache([n], Hkv, D, 0, 412)
    q, kb, vb = (W.normal(412, x, (1, k, h, D), 1.0) for x, h in (("q", Hq), ("k", Hkv), ("v", Hkv)))
    out = torch.empty(1, k, Hq, D, dtype=torch.bfloat16, device="cuda")
    ws = torch.full((L.deer_block_attn_quant_workspace_bytes(1, k, Hq, Hkv, D, msl),), 255, dtype=torch.uint8, device="cuda")
    L.deer_block_attn_quant(kv, _ids(1), q.cuda(), kb.cuda(), vb.cuda(), out, None, 0, scale, msl, ws)
    check_attention(out, q, kb, vb, okv, [0], 0, scale, None, f"scale {scale}")


def test_attention_of_one_long_sequence_and_few_rows():
    """More chunks than one cluster takes, and more pages than a warp's lanes hold numbers of: clusters whose parts a second
    kernel joins, next to a sequence that leaves whole clusters and chunks without work."""
    from paper_2512_15176_b200 import binding as L
    lengths, k, Hq, Hkv, D = [40000, 37, 9000], 3, 8, 2, 128
    kv, okv = _cache(lengths, Hkv, D, 0, 413)
    q, kb, vb = (W.normal(413, x, (3, k, h, D), 1.0) for x, h in (("q", Hq), ("k", Hkv), ("v", Hkv)))
    for msl in (40000, 600000):                                  # (the larger bound: fewer, longer chunks)
        out = torch.full((3, k, Hq, D), float("nan"), dtype=torch.bfloat16, device="cuda")
        ws = torch.full((L.deer_block_attn_quant_workspace_bytes(3, k, Hq, Hkv, D, msl),), 255, dtype=torch.uint8, device="cuda")
        L.deer_block_attn_quant(kv, _ids(3), q.cuda(), kb.cuda(), vb.cuda(), out, None, 0, 1 / math.sqrt(D), msl, ws)
        assert L.deer_kv_status(kv) == 0
        check_attention(out, q, kb, vb, okv, [0, 1, 2], 0, 1 / math.sqrt(D), None, f"bound {msl}")


@pytest.mark.parametrize("M,K,N,res", [(2, 4096, 16, True), (16, 2064, 256, False), (40, 4096, 256, True), (64, 1040, 4096, False), (100, 1024, 2000, True),
                                       (200, 400, 2448, True), (257, 1168, 2400, False), (1000, 272, 2448, True), (700, 640, 4992, False)])
def test_linear_quant_more_shapes(M, K, N, res):
    """Both sides of the rules that choose a kernel: clusters of two to eight blocks for each row tile, pairs of blocks with
    128 and with 256 weight rows, column groups that do not divide evenly, edges in every direction."""
    test_linear_quant(M, K, N, res)


def test_calls_on_two_streams_at_once():
    """The same calls on two streams, each with outputs and a workspace of its own, give what one stream gives."""
    from paper_2512_15176_b200 import binding as L
    kv, okv = _cache([900, 333], 4, 128, 0, 420)
    dev, _, _ = _linear_inputs(33, 1024, 512, seed=421)
    jobs = []
    for k, Hq in ((2, 16), (32, 32)):
        q, kb, vb = (W.normal(420 + k, x, (2, k, h, 128), 1.0).cuda() for x, h in (("q", Hq), ("k", 4), ("v", 4)))
        for msl in (900, 1 << 20):
            ws = torch.empty(L.deer_block_attn_quant_workspace_bytes(2, k, Hq, 4, 128, msl), dtype=torch.uint8, device="cuda")
            jobs.append((q, kb, vb, msl, ws))
    act = W.normal(422, "x", (64, 1024), 1.0).cuda()

    def run(mine):
        outs = []
        for q, kb, vb, msl, ws in mine:
            outs.append(torch.empty_like(q))
            L.deer_block_attn_quant(kv, _ids(2), q, kb, vb, outs[-1], None, 0, 0.088, msl, ws)
        y = torch.empty(33, 512, dtype=torch.bfloat16, device="cuda")
        L.deer_linear_quant(*dev, y)
        codes, scales = torch.empty(64, 1024, dtype=F8, device="cuda"), torch.empty(64, 8, device="cuda")
        L.deer_quantize(act, codes, scales)
        return outs + [y, codes.view(torch.uint8), scales]

    want = run(jobs)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    own = [jobs, [(q, kb, vb, msl, torch.empty_like(ws)) for q, kb, vb, msl, ws in jobs]]
    got = [[], []]
    for _ in range(3):
        for i, st in enumerate(streams):
            st.wait_stream(torch.cuda.current_stream())
            with torch.cuda.stream(st):
                got[i].append(run(own[i]))
    torch.cuda.synchronize()
    assert L.deer_kv_status(kv) == 0
    for runs in got:
        for outs in runs:
            assert all(torch.equal(a, b) for a, b in zip(outs, want))


@pytest.mark.parametrize("k", [2, 32])
def test_the_same_sequence_twice_and_padding_entries(k):
    """Reading calls may name a sequence twice; an entry that names none (padding) is reported and its rows stay."""
    from paper_2512_15176_b200 import binding as L
    kv, okv = _cache([300, 45], 2, 128, 0, 423)
    ids = [1, 0, 0, -1]
    q, kb, vb = (W.normal(423, x, (4, k, h, 128), 1.0) for x, h in (("q", 8), ("k", 2), ("v", 2)))
    for msl in (300, 1 << 20):
        out = torch.full((4, k, 8, 128), 5.0, dtype=torch.bfloat16, device="cuda")
        ws = torch.full((L.deer_block_attn_quant_workspace_bytes(4, k, 8, 2, 128, msl),), 255, dtype=torch.uint8, device="cuda")
        L.deer_block_attn_quant(kv, torch.tensor(ids, dtype=torch.int32, device="cuda"), q.cuda(), kb.cuda(), vb.cuda(), out, None, 0, 0.088, msl, ws)
        assert L.deer_kv_status(kv) == L.DEER_ERR_INVALID_ARG
        check_attention(out[:3], q[:3], kb[:3], vb[:3], okv, ids[:3], 0, 0.088, None, f"bound {msl}")
        assert (out[3] == 5).all()


def test_two_recorded_graphs_share_a_workspace():
    """Two graphs recorded with the same workspace, replayed in turn on one stream."""
    from paper_2512_15176_b200 import binding as L
    kv, okv = _cache([2000], 2, 128, 0, 424)
    data = [[W.normal(424 + i, x, (1, 32, h, 128), 1.0) for x, h in (("q", 8), ("k", 2), ("v", 2))] for i in range(2)]
    for msl in (2000, 1 << 20):
        ws = torch.full((L.deer_block_attn_quant_workspace_bytes(1, 32, 8, 2, 128, msl),), 255, dtype=torch.uint8, device="cuda")
        graphs, outs, keep = [], [], []
        for q, kb, vb in data:
            t = [x.cuda() for x in (q, kb, vb)]
            out, ids = torch.zeros(1, 32, 8, 128, dtype=torch.bfloat16, device="cuda"), _ids(1)
            torch.cuda.synchronize()
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g, stream=torch.cuda.Stream()):
                L.deer_block_attn_quant(kv, ids, *t, out, None, 0, 0.088, msl, ws)
            graphs.append(g)
            outs.append(out)
            keep.append((t, ids))
        for _ in range(3):
            for g in graphs:
                g.replay()
        torch.cuda.synchronize()
        for (q, kb, vb), out in zip(data, outs):
            check_attention(out, q, kb, vb, okv, [0], 0, 0.088, None, f"bound {msl}")


def test_quantise_at_the_edges_of_the_quotient():
    """Groups whose scales span fp32's range, and values at e4m3's rounding borders: the codes are those of the
    correctly rounded quotient, bit for bit."""
    from paper_2512_15176_b200 import binding as L
    rng = np.random.default_rng(425)
    M, K = 512, 1024
    x = rng.standard_normal((M, K)).astype(np.float32)
    x *= np.exp2(rng.integers(-126, 127, size=(M, K // 128)).astype(np.float32)).repeat(128, 1)
    ties = np.array([1.0625, 1.1875, 17.0, 18.0, 19.0, 440.0, 2.0 ** -10, 3 * 2.0 ** -10, 464.0, 0.0], dtype=np.float32)
    x[:, :128] = ties[rng.integers(0, len(ties), size=(M, 128))] * np.exp2(rng.integers(-20, 20, size=(M, 1)).astype(np.float32))
    x[:, 0] = 448.0 * np.exp2(np.floor(rng.uniform(-20, 20, size=M))).astype(np.float32)
    t = torch.from_numpy(x).to(torch.bfloat16)
    codes, scales = torch.empty(M, K, dtype=F8, device="cuda"), torch.empty(M, K // 128, device="cuda")
    L.deer_quantize(t.cuda(), codes, scales)
    want_c, want_s = O.quantise_rows(f64(t))
    assert (scales.cpu().numpy() == want_s).all() and (f64(codes) == want_c).all()


def test_a_bf16_cache_as_an_8_bit_one():
    from paper_2512_15176_b200 import binding as L
    cfg = W.StepConfig("conv", 3, 4, 2, 128, 8, 64, 64, (1, 90), seed=426, growth=8)
    lengths = np.array([48, 1, 90])
    lay = W.kv_layout(cfg, lengths)
    kp, vp = W.kv_pools(cfg, lay.num_pages, sigma=1.0)
    kv = L.KVCacheQuant.from_layout(lay, kp, vp)
    z = lambda *s: np.zeros(s)
    okv = O.QuantKV(z(lay.num_pages, 2, 16, 128), z(lay.num_pages, 2, 16, 128), z(lay.num_pages, 2), z(lay.num_pages, 2), z(3, 2, 48, 128),
                    z(3, 2, 48, 128), lay.page_table, np.zeros(3, dtype=np.int64))
    rows = [np.zeros((3, 90, 2, 128)) for _ in range(2)]
    for x, pool in enumerate((kp, vp)):
        for s, n in enumerate(lengths):
            for tok in range(n):
                rows[x][s, tok] = f64(pool[int(lay.page_table[s, tok // 16]), :, tok % 16])
    okv.store([0, 1, 2], rows[0], rows[1], lengths)
    okv.seq_len = lengths
    got = O.QuantKV(f64(kv.k_pool), f64(kv.v_pool), kv.k_scale.cpu().numpy(), kv.v_scale.cpu().numpy(), f64(kv.k_tail), f64(kv.v_tail), lay.page_table, lengths)
    for s in range(3):
        assert all((a == b).all() for a, b in zip(got.gather(s), okv.gather(s)))


def test_rows_past_four_gigabytes():
    """Operands whose last rows lie behind 2^32 bytes and 2^31 elements: those rows against the oracle."""
    from paper_2512_15176_b200 import binding as L
    M, K = 140000, 16384
    x = torch.zeros(M, K, dtype=torch.bfloat16, device="cuda")
    tail = W.normal(430, "x", (2, K), 1.0)
    x[-2:] = tail.cuda()
    codes, scales = torch.empty(M, K, dtype=F8, device="cuda"), torch.empty(M, K // 128, device="cuda")
    L.deer_quantize(x, codes, scales)
    want_c, want_s = O.quantise_rows(f64(tail))
    assert (f64(codes[-2:]) == want_c).all() and (scales[-2:].cpu().numpy() == want_s).all() and (scales[:-2] == 2.0 ** -126).all()
    g = W.normal(430, "g", (K,), 1.0)
    L.deer_rmsnorm_quant(x, g.cuda(), codes, scales, 1e-6)
    check_codes(codes[-2:], scales[-2:], O.rmsnorm(f64(tail), f64(g), 1e-6), 2e-6, "far rows")
    N = 16384
    xs, w64 = torch.ones(M, 1, device="cuda"), W.normal(431, "w", (N, 16), 1.0, dtype=torch.float32)
    wc, ws = O.quantise_weight(f64(w64))
    xr = torch.zeros(M, 16, device="cuda")
    xr[-2:] = torch.arange(32, device="cuda").view(2, 16) % 9 - 4.0
    xr[0] = 1.0
    y = x[:, :N]
    L.deer_linear_quant(xr.to(F8), xs, torch.from_numpy(wc).float().to(F8).cuda(), torch.from_numpy(ws).cuda(), y)
    w64 = O.dequantise_weight(wc, ws)
    for r in (0, M - 2, M - 1):
        want = w64 @ f64(xr[r])
        assert (np.abs(f64(y[r]) - want) <= 2.0 ** -8 * np.abs(want) + 2.0 ** -16 * (np.abs(w64) @ np.abs(f64(xr[r])))).all()
    assert not y[1:-2].any()


@pytest.mark.parametrize("M,K,N,res", [(64, 1680, 384, True), (70, 1680, 272, False), (128, 2048, 1040, True), (40, 144, 16, True), (48, 1536, 4112, False),
                                       (64, 1024, 9600, True)])
def test_linear_quant_shallow_and_deep(M, K, N, res):
    """More than 32 rows, few tiles: deep products in clusters, shallow ones in one round of pairs."""
    test_linear_quant(M, K, N, res)


def test_rmsnorm_quant_of_extreme_rows():
    """Rows of zeros, of tiny and of huge values next to ordinary ones, and a gain over thirty octaves: codes and scales of
    each row as the oracle has them; a NaN or an infinity spoils its own row and no other."""
    from paper_2512_15176_b200 import binding as L
    M, K = 9, 1040
    x, g = W.normal(440, "x", (M, K), 1.0), W.normal(440, "g", (K,), 1.0)
    g *= torch.exp2((torch.arange(K) % 31 - 15).float()).to(torch.bfloat16)
    x[0] = 0.0
    x[1] *= 2.0 ** -60
    x[2] *= 2.0 ** 50
    x[3, 5] = float("nan")
    x[4, 700] = float("inf")
    x[5, :128] = 0.0
    x[6] = 2.0 ** -100
    codes, scales = torch.empty(M, K, dtype=F8, device="cuda"), torch.empty(M, 9, device="cuda")
    L.deer_rmsnorm_quant(x.cuda(), g.cuda(), codes, scales, 1e-6)
    torch.cuda.synchronize()
    fine = [0, 1, 2, 5, 6, 7, 8]
    check_codes(codes[fine], scales[fine], O.rmsnorm(f64(x[fine]), f64(g), 1e-6), 2e-6, "extreme rows")
    v = codes.float() * scales.repeat_interleave(128, 1)[:, :K]
    assert v[3].isnan().all() and not v[4].isfinite().all() and v[fine].isfinite().all()

"""The verifier layer in 8 bits (runner.VerifierLayerQuant, runner.VerifierStackQuant): every stage against the oracle
on the device's own input of that stage, and several draft-verify steps of a stack over one page table.

Tolerances: those of the single calls (test_gpu_quant); a projection is one bf16 rounding (2^-8 of the value) and at most
2^-16 of its sum of magnitudes."""
import math

import numpy as np
import pytest
import torch

from oracle import deer_oracle as O
from paper_2512_15176_b200 import workload as W
from tests.test_gpu_quant import check_attention, check_codes, f64

pytestmark = pytest.mark.gpu
EPS, THETA = 1e-6, 1.0e6


def _weights(seed, hid, Hq, Hkv, D, inter):
    mk = lambda name, shape, sig: W.normal(seed, name, shape, sig)
    return {"ln1": mk("ln1", (hid,), 1.0), "ln2": mk("ln2", (hid,), 1.0), "q_norm": mk("qn", (D,), 1.0), "k_norm": mk("kn", (D,), 1.0),
            "wqkv": mk("wqkv", ((Hq + 2 * Hkv) * D, hid), hid ** -0.5), "wo": mk("wo", (hid, Hq * D), (Hq * D) ** -0.5),
            "wgu": mk("wgu", (2 * inter, hid), hid ** -0.5), "wd": mk("wd", (hid, inter), inter ** -0.5)}


def _check_linear(y, x, w, residual, label):
    x64 = O.dequantise_rows(f64(x[0]), x[1].cpu().numpy())
    w64 = O.dequantise_weight(f64(w[0]), w[1].cpu().numpy())
    want, mass = x64 @ w64.T, np.abs(x64) @ np.abs(w64).T
    if residual is not None:
        want, mass = want + f64(residual), mass + np.abs(f64(residual))
    err = np.abs(f64(y) - want)
    assert (err <= 2.0 ** -8 * np.abs(want) + 2.0 ** -16 * mass).all(), label


def _check_layer(layer, x, okv, cfg, inter, label):
    M, D = cfg.M, cfg.D
    check_codes(*layer.xn, O.rmsnorm(f64(x), f64(layer.norms["ln1"]), EPS), 2e-6, label + " ln1")
    _check_linear(layer.qkv, layer.xn, layer.w["wqkv"], None, label + " qkv")
    check_attention(layer.attn_out, layer.q, layer.k_blk, layer.v_blk, okv, np.arange(cfg.B), 0, 1 / math.sqrt(D), None, label + " attention")
    codes, scales = O.quantise_rows(f64(layer.attn_out).reshape(M, -1))
    assert (f64(layer.attn_in[0]) == codes).all() and (layer.attn_in[1].cpu().numpy() == scales).all(), label
    _check_linear(layer.x1, layer.attn_in, layer.w["wo"], x, label + " output projection")
    check_codes(*layer.xn2, O.rmsnorm(f64(layer.x1), f64(layer.norms["ln2"]), EPS), 2e-6, label + " ln2")
    _check_linear(layer.gu, layer.xn2, layer.w["wgu"], None, label + " gate and up")
    gu = f64(layer.gu)
    check_codes(*layer.act, O.swiglu(gu[:, :inter], gu[:, inter:]), 8e-6, label + " gated activation")
    _check_linear(layer.x2, layer.act, layer.w["wd"], layer.x1, label + " down projection")


def _empty(cfg, pages, width):
    from paper_2512_15176_b200 import binding as L
    z = lambda *s: np.zeros(s)
    kv = L.KVCacheQuant.empty(pages, cfg.Hkv, cfg.D, cfg.B, width)
    okv = lambda: O.QuantKV(z(pages, cfg.Hkv, 16, cfg.D), z(pages, cfg.Hkv, 16, cfg.D), z(pages, cfg.Hkv), z(pages, cfg.Hkv),
                            z(cfg.B, cfg.Hkv, 48, cfg.D), z(cfg.B, cfg.Hkv, 48, cfg.D), np.zeros((cfg.B, width), dtype=np.int64),
                            np.zeros(cfg.B, dtype=np.int64))
    return kv, okv


def test_weights_are_quantised_by_blocks():
    from paper_2512_15176_b200.runner import quantise_weight
    w = W.normal(600, "w", (200, 336), 0.1)
    w[:128, 256:] = 0.0
    codes, scales = quantise_weight(w.cuda())
    want_c, want_s = O.quantise_weight(f64(w))
    assert (f64(codes) == want_c).all() and (scales.cpu().numpy() == want_s).all()


@pytest.mark.parametrize("B,k,Hq,Hkv,D,hid,inter,prompt", [(3, 8, 8, 2, 128, 512, 1040, 200), (2, 1, 4, 2, 64, 272, 400, 33), (1, 32, 8, 2, 128, 640, 768, 0)])
def test_layer_stages(B, k, Hq, Hkv, D, hid, inter, prompt):
    """A prompt of odd lengths enters the cache, then one block through the layer; the rotary tail bit for bit as the
    same call gives it on a bf16 cache of the same lengths."""
    from paper_2512_15176_b200 import binding as L
    from paper_2512_15176_b200.runner import VerifierLayerQuant
    cfg = W.StepConfig("layerq", B, Hq, Hkv, D, k, hid, 512, (0, prompt), seed=601, growth=k)
    kv, make = _empty(cfg, 80, 24)
    okv = make()
    ids = torch.arange(B, dtype=torch.int32, device="cuda")
    if prompt:
        kr, vr = W.normal(601, "kp", (B, prompt, Hkv, D), 1.0), W.normal(601, "vp", (B, prompt, Hkv, D), 1.0)
        keep = np.array([prompt - 7 * b for b in range(B)])
        kd = torch.tensor(keep, dtype=torch.int32, device="cuda")
        L.deer_kv_reserve_rows(kv, ids, prompt)
        L.deer_kv_store(kv, ids, kr.cuda(), vr.cuda(), kd)
        L.deer_kv_commit_rows(kv, ids, kd, prompt)
        okv.page_table = kv.page_table.cpu().numpy()
        okv.store(np.arange(B), f64(kr), f64(vr), keep)
        okv.seq_len = okv.seq_len + keep
    w = {n: t.cuda() for n, t in _weights(602, hid, Hq, Hkv, D, inter).items()}
    layer = VerifierLayerQuant(cfg, kv, w, prompt + k, inter, EPS, THETA)
    x = W.normal(603, "x", (B * k, hid), 1.0).cuda()
    layer.forward(x)
    torch.cuda.synchronize()
    assert L.deer_kv_status(kv) == 0
    _check_layer(layer, x, okv, cfg, inter, "layer")
    pool = torch.zeros(80, Hkv, 16, D, dtype=torch.bfloat16, device="cuda")
    plain = L.KVCache(pool, pool.clone(), kv.page_table, kv.seq_len, kv.n_pages, kv.free_stack, kv.free_top)
    out = [torch.empty_like(t) for t in (layer.q, layer.k_blk, layer.v_blk)]
    L.deer_qkv_split_norm_rope(plain, ids, layer.qkv, *out, w["q_norm"], w["k_norm"], EPS, THETA)
    assert all(torch.equal(a, b) for a, b in zip(out, (layer.q, layer.k_blk, layer.v_blk)))


def test_stack_over_several_steps_and_in_a_graph():
    """Two layers over one page table, five steps that keep between none and all of their rows: each layer's stages, its
    cache bit by bit, the lengths and the pages.  The same steps replayed from one recorded step (forward, store and
    commit; the lengths change between replays) end in the same caches and outputs, bit for bit."""
    from paper_2512_15176_b200 import binding as L
    from paper_2512_15176_b200.runner import VerifierStackQuant
    B, k, Hq, Hkv, D, hid, inter, steps = 3, 12, 8, 2, 128, 256, 512, 5
    cfg = W.StepConfig("stackq", B, Hq, Hkv, D, k, hid, 512, (0, 64), seed=610, growth=k)
    weights = [{n: t.cuda() for n, t in _weights(611 + l, hid, Hq, Hkv, D, inter).items()} for l in range(2)]
    keeps = np.array([[12, 0, 5], [7, 12, 1], [0, 0, 0], [12, 12, 12], [3, 9, 11]])
    xs = [W.normal(620 + i, "x", (B * k, hid), 1.0).cuda() for i in range(steps)]
    ends = []
    for recorded in (False, True):
        kv, make = _empty(cfg, 24, 6)
        kvs, okvs = [kv, kv.layer()], [make(), make()]
        stack = VerifierStackQuant(cfg, kvs, weights, 6 * 16, inter, EPS, THETA)
        x, keep = torch.empty_like(xs[0]), torch.zeros(B, dtype=torch.int32, device="cuda")
        outs = []
        if recorded:
            graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
            with torch.cuda.graph(graph, stream=side):
                out = stack.forward(x)
                stack.commit(keep)
        for i in range(steps):
            x.copy_(xs[i])
            keep.copy_(torch.from_numpy(keeps[i].astype(np.int32)))
            if recorded:
                graph.replay()
            else:
                out = stack.forward(x)
                table = kv.page_table.cpu().numpy().copy()
                cur = x
                for l, layer in enumerate(stack.layers):
                    okvs[l].page_table = table
                    _check_layer(layer, cur, okvs[l], cfg, inter, f"step {i} layer {l}")
                    cur = layer.x2
                stack.commit(keep)
                for l, layer in enumerate(stack.layers):
                    okvs[l].store(np.arange(B), f64(layer.k_blk), f64(layer.v_blk), keeps[i])
                    okvs[l].seq_len = okvs[l].seq_len + keeps[i]
                    for x_, (pool, scale, tail) in enumerate(((kvs[l].k_pool, kvs[l].k_scale, kvs[l].k_tail), (kvs[l].v_pool, kvs[l].v_scale, kvs[l].v_tail))):
                        assert (f64(pool) == okvs[l].codes[x_]).all() and (scale.cpu().numpy() == okvs[l].scale[x_]).all()
                        assert (f64(tail) == okvs[l].tail[x_]).all()
                assert (kv.seq_len.cpu().numpy() == okvs[0].seq_len).all()
                assert (kv.n_pages.cpu().numpy() == -(-okvs[0].seq_len // 16)).all()
            outs.append(out.clone())
        torch.cuda.synchronize()
        assert all(L.deer_kv_status(c) == 0 for c in kvs)
        ends.append(outs + [kv.seq_len, kv.page_table, kv.free_top] + [t.view(torch.uint8) for c in kvs for t in (c.k_pool, c.v_pool)]
                    + [t for c in kvs for t in (c.k_scale, c.v_scale, c.k_tail, c.v_tail)])
    assert all(torch.equal(a, b) for a, b in zip(*ends))

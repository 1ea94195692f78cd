"""The 8-bit calls at the ends of their ranges, against the oracle in 64 bits (tolerances as in test_gpu_quant)."""
import math

import numpy as np
import pytest
import torch

from oracle import deer_oracle as O
from paper_2512_15176_b200 import workload as W
from tests.test_gpu_quant import F8, _cache, _ids, check_attention, check_codes, f64

pytestmark = pytest.mark.gpu


GATES = [s * 2.0 ** e for s in (1.0, -1.0) for e in range(-133, 128)] + \
    [-60.0, -69.0, -70.0, -75.0, -80.0, -87.0, -87.5, -88.0, -88.5, -89.0, -95.0, -100.0, -103.0, -104.0, -173.0, -175.0, -200.0, -253.0, -400.0, -1e4, -1e20,
     -1e27, -1e30, -3e38, 2.3e38, 2.4e38, 3e38, torch.finfo(torch.bfloat16).max, torch.finfo(torch.bfloat16).min, 0.0, -0.0]


def _gated(x):
    """Device codes and scales of gated rows x [M, 2 K], and the definition in 64 bits."""
    from paper_2512_15176_b200 import binding as L
    M, K = x.shape[0], x.shape[1] // 2
    codes, scales = torch.empty(M, K, dtype=F8, device="cuda"), torch.empty(M, -(-K // 128), device="cuda")
    L.deer_quantize(x.cuda(), codes, scales, gated=True)
    x64 = f64(x)
    with np.errstate(over="ignore"):                       # exp(-v) = inf: the quotient is 0
        y = x64[:, :K] / (1.0 + np.exp(-x64[:, :K])) * x64[:, K:]
    return f64(codes), scales.cpu().numpy().astype(np.float64), y


def _check_gated(got, s, y, label):
    """As test_gpu_quant.check_codes; and where a gated value is subnormal, it has been rounded four times to a multiple of 2^-149
    (two steps of the numerator, the quotient, the product with up <= 8 in magnitude): 2^-145 / 2^-126 in a code's quotient."""
    delta = 8e-6
    amax = np.abs(y).reshape(y.shape[0], -1, 128).max(axis=2)
    want_s = np.maximum(amax / 448.0, 2.0 ** -126)
    assert (np.abs(s - want_s) <= 2 * delta * want_s).all(), label
    q = np.clip(y / want_s.repeat(128, 1), -448, 448)
    tol = O.e4m3_step(q) / 2 + 4 * delta * np.abs(q) + 2.0 ** -18
    assert np.isfinite(got).all() and (np.abs(got - q) <= tol).all(), f"{label}: {np.max(np.abs(got - q) - tol)}"


def test_gates_of_every_size_alone_in_their_group():
    """A row per gate value, which fills its group: scales and codes follow v / (1 + exp(-v)) * u over all of bf16's exponents."""
    x = torch.empty(len(GATES), 256, dtype=torch.bfloat16)
    x[:, :128] = torch.tensor(GATES)[:, None].to(torch.bfloat16)
    u = W.normal(450, "u", (len(GATES), 128), 1.0).clamp(-0.98, 0.98)
    x[:, 128:] = u
    _check_gated(*_gated(x), "alone")


def test_one_far_gate_leaves_its_neighbours_their_codes():
    """A strongly negative gate among ordinary ones is a zero among them: the group's scale is the ordinary values'."""
    far = [v for v in GATES if v <= -60.0]
    x = W.normal(451, "x", (len(far), 512), 2.0).clamp(-7.9, 7.9)
    x[:, 37] = torch.tensor(far).to(torch.bfloat16)
    x[:, 130] = torch.finfo(torch.bfloat16).min
    x[:, 255] = -1e30
    _check_gated(*_gated(x), "among others")


def test_gated_groups_of_zeros_nan_and_infinities():
    """A NaN or an infinity, as a gate or as the value that it gates, spoils its own group of 128 columns and no other."""
    x = W.normal(452, "x", (7, 1024), 1.0)
    x[0, :128] = 0.0                                       # gates of zero
    x[0, 640:768] = 0.0                                    # values of zero
    bad = {1: (3, float("nan")), 2: (130, float("inf")), 3: (260, -float("inf")), 4: (512 + 5, float("nan")), 5: (512 + 140, float("inf")),
           6: (512 + 390, -float("inf"))}
    for m, (c, v) in bad.items():
        x[m, c] = v
    clean = x.clone()
    for m, (c, v) in bad.items():
        clean[m, c] = 0.0
    got, s, _ = _gated(x)
    _, _, y = _gated(clean)
    for m, (c, v) in bad.items():
        g = c % 512 // 128
        assert not np.isfinite(got[m, g * 128:(g + 1) * 128] * s[m, g]).any()
        got[m, g * 128:(g + 1) * 128], s[m, g], y[m, g * 128:(g + 1) * 128] = 0.0, 2.0 ** -126, 0.0
    _check_gated(got, s, y, "the other groups")


@pytest.mark.parametrize("K", [64, 1040, 4096, 6000, 8208, 20000])
def test_rows_whose_squares_leave_fp32(K):
    """Rows so large, or with eps 0 so small, that the sum of their squares is beyond fp32: the normalised row is an ordinary one."""
    from paper_2512_15176_b200 import binding as L
    M, G = 8, -(-K // 128)
    x, g = W.normal(453, "x", (M, K), 1.0), W.normal(453, "g", (K,), 1.0)
    x[0] *= 2.0 ** 62
    x[1] *= 2.0 ** 70
    x[2] *= 2.0 ** 124
    x[3, 7] = torch.finfo(torch.bfloat16).max
    x[4] *= 2.0 ** -40
    x[5] *= 2.0 ** -75
    x[6] *= 2.0 ** -115
    r = torch.zeros_like(x)
    r[3] = W.normal(453, "r", (1, K), 1.0)[0] * 2.0 ** 115
    for eps, rows, res in ((1e-6, [0, 1, 2, 3, 7], True), (0.0, list(range(M)), False)):
        codes, scales = torch.empty(M, K, dtype=F8, device="cuda"), torch.empty(M, G, device="cuda")
        dev = x.cuda()
        tot = torch.empty_like(dev) if res else dev        # (in place as well)
        L.deer_rmsnorm_quant(dev, g.cuda(), codes, scales, eps, residual=r.cuda() if res else None, total=tot)
        h = f64(x) + (f64(r) if res else 0.0)
        with np.errstate(over="ignore"):
            h32 = h.astype(np.float32)
        assert (f64(tot) == f64(torch.from_numpy(h32).to(torch.bfloat16))).all()
        check_codes(codes[rows], scales[rows], O.rmsnorm(h[rows], f64(g), eps), 2e-6, f"eps {eps}")


def _attend(kv, q, kb, vb, msl, mask=0, states=None):
    from paper_2512_15176_b200 import binding as L
    B, k, Hq, D = q.shape
    out = torch.full((B, k, Hq, D), float("nan"), dtype=torch.bfloat16, device="cuda")
    ws = torch.full((L.deer_block_attn_quant_workspace_bytes(B, k, Hq, kv.n_kv_heads, D, msl),), 255, dtype=torch.uint8, device="cuda")
    L.deer_block_attn_quant(kv, _ids(B), q.cuda(), kb.cuda(), vb.cuda(), out, None if states is None else torch.from_numpy(states).cuda(), mask,
                            1 / math.sqrt(D), msl, ws)
    assert L.deer_kv_status(kv) == 0
    return out


def _block(seed, k, Hq, Hkv, D=128):
    return [W.normal(seed, n, (1, k, h, D), 1.0) for n, h in (("q", Hq), ("k", Hkv), ("v", Hkv))]


BOUNDS = pytest.mark.parametrize("long", [False, True])            # True: the tensor-memory kernel, whatever the lengths are


@BOUNDS
@pytest.mark.parametrize("n", [0, 40, 200])
@pytest.mark.parametrize("octaves", [-30, -60, 30])
def test_values_of_any_magnitude(n, octaves, long):
    """All values scaled by one power of two scale the result, whichever tile comes first and however many tokens the last holds."""
    kv, okv = _cache([n], 2, 128, 0, 460)
    okv.scale[1] *= np.float32(2.0 ** octaves)
    okv.tail[1] *= 2.0 ** octaves
    kv.v_scale.mul_(2.0 ** octaves)
    kv.v_tail.mul_(2.0 ** octaves)
    q, kb, vb = _block(460, 32, 8, 2)
    vb *= 2.0 ** octaves
    check_attention(_attend(kv, q, kb, vb, 1 << 20 if long else n), q, kb, vb, okv, [0], 0, 1 / math.sqrt(128), None, f"{n} 2^{octaves}")


@BOUNDS
@pytest.mark.parametrize("k,Hq,Hkv", [(32, 8, 2), (4, 4, 2)])
@pytest.mark.parametrize("at,lift", [(0, 0.0), (20, 0.0), (0, 30.0), (0, -30.0)])
@pytest.mark.parametrize("octaves", [30, 60])
def test_a_page_of_large_values_and_little_weight(at, lift, octaves, k, Hq, Hkv, long):
    """Page `at` has values 2^octaves times the others', and weights so small that it adds a part of the result that is about as
    large as the others' or far smaller.  The scores behind the first four pages lie `lift` above those of the first four."""
    n, D = 640, 128
    kv, okv = _cache([n], Hkv, D, 0, 461)
    q, kb, vb = _block(461, k, Hq, Hkv)
    q = q * 0.05
    q[..., 0] = 8.0                                        # dim 0 carries the level of a page's scores
    key = lambda level: level * math.sqrt(D) / 8.0
    okv.scale[0][:] = 0.5
    K = O.e4m3_round(np.clip(okv.codes[0] / 30.0, -4.0, 4.0))
    for p in range(n // 16):
        level = -(octaves * math.log(2.0) + 1.0) if p == at else lift if p >= 4 else 0.0
        K[okv.page_table[0, p], :, :, 0] = O.e4m3_round(key(level) / 0.5)
    okv.codes[0] = K
    okv.scale[1][okv.page_table[0, at]] *= np.float32(2.0 ** octaves)
    kb[..., 0] = key(max(lift, 0.0))
    kv.k_pool.copy_(torch.from_numpy(okv.codes[0]).float().to(F8))
    kv.k_scale.copy_(torch.from_numpy(okv.scale[0]))
    kv.v_scale.copy_(torch.from_numpy(okv.scale[1]))
    check_attention(_attend(kv, q, kb, vb, 1 << 20 if long else n), q, kb, vb, okv, [0], 0, 1 / math.sqrt(D), None, f"page {at}")


@BOUNDS
@pytest.mark.parametrize("k,Hq,Hkv", [(32, 16, 4), (20, 8, 1), (4, 4, 2)])
@pytest.mark.parametrize("size", [2.0 ** 20, 2.0 ** 40, torch.finfo(torch.bfloat16).max, torch.finfo(torch.bfloat16).min])
@pytest.mark.parametrize("what", ["key", "value"])
def test_large_finite_rows_reach_only_rows_that_see_them(what, size, k, Hq, Hkv, long):
    """The last draft row, which the rows before it do not see, has a key or a value of any finite size."""
    n, D = 200, 128
    kv, okv = _cache([n], Hkv, D, 0, 462)
    q, kb, vb = _block(462, k, Hq, Hkv)
    clean = [t.clone() for t in (q, kb, vb)]
    without = _attend(kv, q, kb, vb, 1 << 20 if long else n)
    (kb if what == "key" else vb)[0, k - 1] = size
    out = _attend(kv, q, kb, vb, 1 << 20 if long else n)
    assert torch.equal(out[:, :-1], without[:, :-1])
    check_attention(out[:, :-1], *[t[:, :-1] for t in clean], okv, [0], 0, 1 / math.sqrt(D), None, what)
    # as a row that is still masked, the decoded rows do not see it either
    states = np.zeros((1, k), dtype=np.int32)
    states[0, -1] = 1
    out = _attend(kv, q, kb, vb, 1 << 20 if long else n, 1, states)
    st = states.copy()
    st[0, -1] = -1
    want = _attend(kv, clean[0], clean[1], clean[2], 1 << 20 if long else n, 1, st)
    assert torch.equal(out[:, :-1], want[:, :-1])


@BOUNDS
@pytest.mark.parametrize("k,Hq,Hkv", [(32, 16, 4), (4, 4, 2)])
def test_tail_and_block_rows_of_very_different_size(k, Hq, Hkv, long):
    """Neighbouring tokens whose keys and values differ by many octaves in size; the largest keys lie across the queries, so that the
    smaller ones' scores decide."""
    n, D = 206, 128
    kv, okv = _cache([n], Hkv, D, 0, 463)
    q, kb, vb = _block(463, k, Hq, Hkv)
    q[..., 5] = 0.0
    kb[:, ::5] = 0.0
    kb[:, ::5, :, 5] = 2.0 ** 30
    okv.tail[0][:, :, 1::5] = 0.0
    okv.tail[0][:, :, 1::5, 5] = -2.0 ** 25
    vb[:, ::7] *= 2.0 ** -20
    okv.tail[1][:, :, ::3] *= 2.0 ** -40
    kv.k_tail.copy_(torch.from_numpy(okv.tail[0]).to(torch.bfloat16))
    kv.v_tail.copy_(torch.from_numpy(okv.tail[1]).to(torch.bfloat16))
    check_attention(_attend(kv, q, kb, vb, 1 << 20 if long else n), q, kb, vb, okv, [0], 0, 1 / math.sqrt(D), None, "sizes")


@BOUNDS
@pytest.mark.parametrize("k,Hq,Hkv", [(32, 8, 2), (4, 4, 2)])
@pytest.mark.parametrize("which,bad", [("k_scale", float("nan")), ("v_scale", float("nan")), ("v_scale", float("inf"))])
def test_a_page_scale_that_is_not_finite(which, bad, k, Hq, Hkv, long):
    """Every row of the page's head sees the page, and no row of another head does."""
    kv, okv = _cache([330], Hkv, 128, 0, 464)
    q, kb, vb = _block(464, k, Hq, Hkv)
    getattr(kv, which)[int(okv.page_table[0, 9]), 1] = bad
    out = _attend(kv, q, kb, vb, 1 << 20 if long else 330)
    G = Hq // Hkv
    assert not out[:, :, G:].isfinite().any()
    fine = [t[:, :, :1] for t in (kb, vb)]
    one = O.QuantKV(*[c[:, :1] for c in okv.codes], *[c[:, :1] for c in okv.scale], *[c[:, :1] for c in okv.tail], okv.page_table, okv.seq_len)
    check_attention(out[:, :, :G], q[:, :, :G], *fine, one, [0], 0, 1 / math.sqrt(128), None, which)

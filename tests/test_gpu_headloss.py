"""The LM head's losses, their gradients and the top logits on the GPU against the 64-bit oracle.

Tolerances (u = 2^-24, half a step of fp32; b = 2^-8, half a step of bf16):
* z: hid / 16 instructions add to an fp32 accumulator, each off by at most two half steps of the sum of magnitudes, and a few
  more inside one: dz = (hid / 16 + 8) 2u sum |h w|.
* lse: dz / tau, and 2^-20 for the exponentials, their sum and the logarithm, and 8u of its size.
* loss: tau^2 a times (2 dz / tau + 2^-20 + 16u (|lse| + max |z| / tau + max |log t|)), in the list's mean.
* G: rounded once to bf16, b |G| (b^2 |G| where it is held as two terms: up to 128
  live rows for dh, 64 for dw); p off by the factor d = 2 dz / tau + 2^-19; 8u of t.
* dh, dw: G's errors against |w| (|h|), the accumulator's (n / 16 + 8) 2u of sum |G w| over n terms, and one rounding b."""
import math

import numpy as np
import pytest
import torch

from oracle import deer_oracle as O

pytestmark = pytest.mark.gpu
U, B = 2.0 ** -24, 2.0 ** -8


@pytest.fixture(scope="module")
def L():
    from paper_2512_15176_b200 import binding
    binding.lib()
    return binding


def f64(t):
    return t.double().cpu().numpy()


def draw(seed, M, hid, V, K=None, live=1.0, sure=8.0, spread=1.0):
    """Hidden states that favour their first target by up to `sure`; a share `live` of the rows has a target."""
    g = torch.Generator().manual_seed(seed)
    n = K or 1
    w = (spread * torch.randn(V, hid, generator=g) / math.sqrt(hid)).bfloat16()
    ids = torch.stack([torch.randperm(V, generator=g)[:n] if V >= n else torch.randint(V, (n,), generator=g) for _ in range(M)]).int()
    best = w[ids[:, 0].long()].float()
    h = (torch.randn(M, hid, generator=g) + sure * torch.rand(M, 1, generator=g) * best / best.square().sum(1, keepdim=True).clamp_min(1e-3)).bfloat16()
    ids[torch.rand(M, generator=g) >= live] = -1
    teacher = (3 * torch.randn(M, n, generator=g)).sort(dim=1, descending=True).values if K else None
    return h, w, ids, teacher, 0.5 + torch.rand(M, generator=g), torch.randn(M, generator=g) / M


def run(L, h, w, ids, teacher=None, tau=1.0, weight=None, grad=None, dh=True, dw=True, ws=None):
    M, hid = h.shape
    V, K = w.shape[0], ids.shape[1]
    c = lambda t: None if t is None else t.cuda().contiguous()  # noqa: E731
    h, w, ids, teacher, weight, grad = (c(t) for t in (h, w, ids, teacher, weight, grad))
    o = lambda *s, dtype=torch.float32: torch.full(s, 7.0, dtype=dtype, device="cuda")  # noqa: E731
    loss, lse, tl = o(M), o(M), o(M, K)
    dh, dw = o(M, hid, dtype=torch.bfloat16) if dh else None, o(V, hid, dtype=torch.bfloat16) if dw else None
    # a workspace of its own for each call, full of NaN: nothing in it may count
    space = lambda g: torch.full((L.deer_lmhead_loss_workspace_bytes(M, hid, V, K, g) + 16,), 255, dtype=torch.uint8, device="cuda")  # noqa: E731
    if teacher is None:
        L.deer_lmhead_loss(h, w, ids[:, 0].contiguous(), loss, lse, tl[:, 0].contiguous() if K > 1 else tl, space(False), weight)
        if dh is not None or dw is not None:
            L.deer_lmhead_loss_grad(h, w, ids[:, 0].contiguous(), lse, tl, dh, dw, space(True), weight, grad)
    else:
        L.deer_lmhead_distill(h, w, ids, teacher, tau, loss, lse, tl, space(False), weight)
        if dh is not None or dw is not None:
            L.deer_lmhead_distill_grad(h, w, ids, teacher, tau, lse, tl, dh, dw, space(True), weight, grad)
    torch.cuda.synchronize()
    return loss, lse, tl, dh, dw


def check(got, h, w, ids, teacher=None, tau=1.0, weight=None, grad=None):
    h, w, ids = f64(h), f64(w), ids.cpu().numpy()
    teacher, weight, grad = (None if t is None else f64(t) for t in (teacher, weight, grad))
    M, hid = h.shape
    V = w.shape[0]
    loss, lse, tl, dh, dw = got
    want, want_lse, p, t, live = O.head_loss(h, w, ids, teacher, tau, weight)
    aw = np.abs(w)
    dz = (hid / 16 + 8) * 2 * U * (np.abs(h) @ aw.T).max(axis=1) * live
    z = h @ w.T
    a = np.ones(M) if weight is None else np.abs(weight)
    size = np.abs(want_lse) + np.abs(z).max(axis=1) / tau + (0 if teacher is None else np.where(np.isfinite(teacher), np.abs(teacher), 0).max(axis=1) * 2 / tau + 5)
    assert (np.abs(f64(lse) - want_lse) <= dz / tau + 2.0 ** -20 + 8 * U * np.abs(want_lse)).all(), np.abs(f64(lse) - want_lse).max()
    tol = tau ** 2 * a * (2 * dz / tau + 2.0 ** -20 + 16 * U * size)
    assert (np.abs(f64(loss) - want) <= tol).all(), (np.abs(f64(loss) - want) / tol).max()
    assert (f64(loss)[~live] == 0).all() and (f64(lse)[ids[:, 0] < 0] == 0).all()
    for m in range(M):                                                        # the listed tokens' z, 0 behind the end
        n = int(np.argmax(np.append(ids[m], -1) < 0)) if live[m] else 0
        zt = f64(tl)[m]
        assert (zt[n:] == 0).all() or not live[m]
        assert (np.abs(zt[:n] - z[m, ids[m, :n]]) <= dz[m]).all()
    want_dh, want_dw, G = O.head_loss_grad(h, w, ids, teacher, tau, weight, grad)
    c = np.abs((1 if weight is None else weight) * (1 if grad is None else grad) * tau * live)[:, None] * np.ones((M, 1))
    dp = c * (p * (2 * dz / tau + 2.0 ** -19)[:, None] + 8 * U * t)
    for x, want_x, other, n in ((dh, want_dh, aw, V), (dw, want_dw, np.abs(np.where(live[:, None], h, 0)), M)):
        if x is None:
            continue
        dG = (B if live.sum() > (128 if x is dh else 64) else B * B) * np.abs(G) + dp
        d, s = (dG @ other, np.abs(G) @ other) if x is dh else (dG.T @ other, np.abs(G).T @ other)
        tol = B * np.abs(want_x) + (1 + B) * (d + (n / 16 + 8) * 2 * U * s) + 2.0 ** -133
        err = np.abs(f64(x) - want_x)
        assert (err <= tol).all(), ((err / tol).max(), np.unravel_index((err / tol).argmax(), err.shape))


SHAPES = [(1, 64, 16), (1, 64, 1), (3, 128, 33), (8, 512, 4096), (33, 192, 1000), (127, 320, 515), (129, 64, 300), (256, 128, 257), (257, 576, 801),
          (300, 256, 5003), (700, 64, 130), (40, 2048, 600)]


@pytest.mark.parametrize("M,hid,V", SHAPES)
@pytest.mark.parametrize("live", [1.0, 0.5])
def test_cross_entropy(L, M, hid, V, live):
    h, w, ids, _, a, g = draw(M * 7 + V, M, hid, V, live=live)
    check(run(L, h, w, ids, weight=a, grad=g), h, w, ids, weight=a, grad=g)


@pytest.mark.parametrize("M,hid,V", [(2, 64, 40), (130, 192, 900), (257, 128, 700)])
def test_weights_and_upstream_default_to_one(L, M, hid, V):
    h, w, ids, _, a, g = draw(3, M, hid, V, live=0.8)
    check(run(L, h, w, ids), h, w, ids)
    check(run(L, h, w, ids, weight=a, dw=False), h, w, ids, weight=a)
    check(run(L, h, w, ids, grad=g, dh=False), h, w, ids, grad=g)


@pytest.mark.parametrize("M,hid,V,K,tau", [(1, 64, 50, 1, 1.0), (4, 128, 200, 8, 1.0), (33, 192, 1000, 32, 2.0), (65, 64, 333, 33, 0.7), (130, 256, 900, 64, 1.0),
                                           (260, 128, 700, 128, 1.5), (20, 512, 4099, 127, 1.0)])
def test_distillation(L, M, hid, V, K, tau):
    h, w, ids, teacher, a, g = draw(M + K, M, hid, V, K=K, live=0.9)
    length = torch.randint(1, K + 1, (M, 1), generator=torch.Generator().manual_seed(K))
    ids[torch.arange(K)[None, :] >= length] = -1
    args = dict(teacher=teacher, tau=tau, weight=a, grad=g)
    check(run(L, h, w, ids, **args), h, w, ids, **args)


def test_lists_with_repeats_gaps_and_neighbours(L):
    M, hid, V, K = 12, 128, 600, 6
    h, w, ids, teacher, a, g = draw(9, M, hid, V, K=K)
    ids[0] = 17                                                               # one token, six times
    ids[1, 3] = ids[1, 0]
    ids[2, 2:] = torch.tensor([-1, 5, 6, 7])                                  # behind the end: not looked at
    ids[3] = torch.arange(V - K, V)                                           # the vocabulary's last tokens
    ids[4] = torch.tensor([255, 256, 63, 64, 191, 192])                       # the borders of tiles and chunks
    ids[5] = torch.arange(5, -1, -1)
    teacher[6, 1:] = -math.inf                                                # one token left
    teacher[7] = -math.inf                                                    # no distribution
    teacher[8, 0] = 200.0                                                     # all but one underflow
    teacher[9] = torch.finfo(torch.float32).min                               # the type's lowest value, all alike
    a[10] = 0.0
    args = dict(teacher=teacher, tau=1.0, weight=a, grad=g)
    got = run(L, h, w, ids, **args)
    check(got, h, w, ids, **args)
    assert got[0][7] == 0 and got[0][10] == 0 and not got[3][7].any() and not got[3][10].any()


def test_no_row_is_live(L):
    for M, hid, V in ((1, 64, 20), (70, 128, 400)):
        h, w, ids, _, a, g = draw(1, M, hid, V, live=0.0)
        loss, lse, tl, dh, dw = run(L, torch.full_like(h, math.nan), w, ids, weight=a, grad=g)
        for t in (loss, lse, tl, dh, dw):
            assert (t == 0).all()
        loss, _, _, dh, dw = run(L, h, w, ids.abs(), weight=torch.zeros(M))
        assert (loss == 0).all() and (dh == 0).all() and (dw == 0).all()


def test_dead_rows_may_hold_anything(L):
    h, w, ids, _, a, g = draw(5, 150, 128, 500, live=0.5)
    dead = ids[:, 0] < 0
    clean = run(L, h, w, ids, weight=a, grad=g)
    h2, a2, g2 = h.clone(), a.clone(), g.clone()
    h2[dead], a2[dead], g2[dead] = math.nan, math.inf, math.nan
    for x, y in zip(clean, run(L, h2, w, ids, weight=a2, grad=g2)):
        assert torch.equal(x, y)
    a2[~dead & (torch.arange(150) % 3 == 0)] = 0.0                            # and rows of weight 0
    some = ids.clone()
    some[a2 == 0] = -1
    h2[a2 == 0] = math.inf
    for x, y in zip(run(L, h, w, some, weight=a, grad=g), run(L, h2, w, ids, weight=a2, grad=g2)):
        assert torch.equal(x, y)


def test_a_row_that_is_not_finite_stays_alone_in_dh(L):
    h, w, ids, _, a, g = draw(6, 40, 128, 500)
    clean = run(L, h, w, ids, weight=a, grad=g)
    h2 = h.clone()
    h2[7, 3] = math.nan
    loss, lse, tl, dh, dw = run(L, h2, w, ids, weight=a, grad=g)
    keep = torch.arange(40) != 7
    assert torch.isnan(loss[7]) and torch.isnan(lse[7]) and torch.isnan(dh[7]).all() and torch.isnan(dw).all()
    assert torch.equal(loss[keep], clean[0][keep]) and torch.equal(dh[keep], clean[3][keep])


def test_tokens_outside_the_vocabulary(L):
    M, hid, V, K = 30, 128, 500, 4
    h, w, ids, teacher, a, g = draw(8, M, hid, V, K=K)
    out = ids.clone()
    out[3, 2], out[11, 0], out[12, 3] = V, 2 ** 31 - 1, V + 5
    bad = torch.zeros(M, dtype=torch.bool)
    bad[[3, 11, 12]] = True
    got = run(L, h, w, out, teacher=teacher, tau=1.0, weight=a, grad=g)
    assert torch.isnan(got[0][bad]).all() and torch.isfinite(got[0][~bad]).all()
    assert (got[3][bad] == 0).all()
    a0 = a.clone()
    a0[bad] = 0.0                                                             # the gradient of the others
    want = run(L, h, w, ids, teacher=teacher, tau=1.0, weight=a0, grad=g)
    torch.testing.assert_close(got[4].float(), want[4].float(), rtol=0, atol=float(2 * B * want[4].abs().max()))
    assert torch.equal(got[3][~bad], want[3][~bad])
    one = run(L, h, w, torch.where(bad[:, None], V, ids)[:, :1].contiguous(), weight=a, grad=g)
    assert torch.isnan(one[0][bad]).all() and torch.isfinite(one[0][~bad]).all() and (one[3][bad] == 0).all() and torch.isfinite(one[4]).all()


def test_large_logits_and_sure_rows(L):
    # logits of hundreds: probabilities of exactly 1 and 0, and targets that the model is all but sure of
    h, w, ids, _, a, g = draw(12, 64, 256, 800, sure=400.0)
    check(run(L, h, w, ids, weight=a, grad=g), h, w, ids, weight=a, grad=g)
    h, w, ids, _, a, g = draw(13, 64, 256, 800, sure=24.0)
    check(run(L, h, w, ids, weight=a, grad=g), h, w, ids, weight=a, grad=g)


def test_several_pieces_of_the_vocabulary(L):
    # 4096 rows: pieces of 32768 tokens at most; some live rows, an odd end.  The oracle in 64 bits on the device.
    M, hid, V, K = 4096, 64, 70001, 3
    g = torch.Generator(device="cuda").manual_seed(3)
    r = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
    w, h = (r(V, hid) / 8).bfloat16(), r(M, hid).bfloat16()
    ids = torch.randint(V, (M, K), generator=g, device="cuda").int()
    ids[:, 1:] = torch.where(ids[:, 1:] == ids[:, :1], (ids[:, 1:] + 1) % V, ids[:, 1:])
    ids[100:2500] = -1
    teacher, a = r(M, K), torch.rand(M, generator=g, device="cuda") + 0.5
    loss, lse, tl, dh, dw = run(L, h, w, ids, teacher=teacher, tau=1.0, weight=a)
    live = ids[:, 0] >= 0
    z = h[live].double() @ w.double().T
    t = torch.softmax(teacher[live].double(), 1)
    logp = torch.log_softmax(z, 1)
    want = a[live] * (t * (torch.log(t) - torch.gather(logp, 1, ids[live].long()))).sum(1)
    dz = (hid / 16 + 8) * 2 * U * (h[live].double().abs() @ w.double().abs().T).amax(1)
    tol = a[live] * (2 * dz + 2.0 ** -20 + 16 * U * 40)
    assert ((loss[live] - want).abs() <= tol).all() and (loss[~live] == 0).all() and (dh[~live] == 0).all()
    G = torch.exp(logp)
    G.scatter_add_(1, ids[live].long(), -t)
    G *= a[live].double()[:, None]
    dG = B * G.abs() + a[live].double()[:, None] * torch.exp(logp) * (2 * dz[:, None] + 2.0 ** -19) + 1e-6 * (G < 0)
    for x, want_x, other, f in ((dh[live], G @ w.double(), w.double().abs(), lambda e: e), (dw, G.T @ h[live].double(), h[live].double().abs(), lambda e: e.T)):
        tol = B * want_x.abs() + (1 + B) * (f(dG) @ other + (V / 16 + 8) * 2 * U * (f(G.abs()) @ other))
        assert ((x.double() - want_x).abs() <= tol).all()
        rel = ((x.double() - want_x).norm() / want_x.norm()).item()
        assert rel < 2 * B, rel                                               # two roundings, never all at their worst


def test_same_bits_every_time(L):
    h, w, ids, teacher, a, g = draw(21, 300, 256, 5000, K=16, live=0.7)
    first = run(L, h, w, ids, teacher=teacher, tau=1.3, weight=a, grad=g)
    for _ in range(3):
        for x, y in zip(first, run(L, h, w, ids, teacher=teacher, tau=1.3, weight=a, grad=g)):
            assert torch.equal(x, y)


# ---------------------------------------------------------------------------------------------------------------
# top logits
# ---------------------------------------------------------------------------------------------------------------

def top(L, z, K):
    z = z.cuda().contiguous()
    ids = torch.full((z.shape[0], K), 99, dtype=torch.int32, device="cuda")
    values = torch.full((z.shape[0], K), 99.0, device="cuda")
    L.deer_top_logits(z, ids, values)
    torch.cuda.synchronize()
    return ids.cpu(), values.cpu()


def check_top(L, z, K):
    ids, values = top(L, z, K)
    n = min(K, z.shape[1])
    if torch.isnan(z).any():
        want_ids, want = O.top_logits(z.numpy(), K)
        np.testing.assert_array_equal(ids.numpy(), want_ids)
        np.testing.assert_array_equal(values.numpy(), want)
        return
    want = torch.sort(z + 0.0, dim=1, descending=True, stable=True).indices[:, :n].int()
    assert torch.equal(ids[:, :n], want)
    assert torch.equal(values[:, :n], torch.gather(z, 1, want.long()))
    assert (ids[:, n:] == -1).all() and (values[:, n:] == -math.inf).all()


@pytest.mark.parametrize("M,V", [(1, 1), (2, 7), (3, 100), (1, 4096), (2, 4097), (5, 5001), (1, 8192), (9, 8195), (1, 32768), (40, 33001), (1, 151936),
                                 (3, 151937), (160, 20001), (300, 9999)])
@pytest.mark.parametrize("K", [1, 8, 50, 128])
def test_top_logits(L, M, V, K):
    check_top(L, 3 * torch.randn(M, V, generator=torch.Generator().manual_seed(V + K)), K)


@pytest.mark.parametrize("V", [3000, 5003, 40000, 151936])
def test_top_logits_of_unlike_rows(L, V):
    g = torch.Generator().manual_seed(V)
    n = torch.randn(V, generator=g)
    rows = [torch.zeros(V), -torch.arange(V).float(), torch.arange(V).float(), torch.round(n * 2), torch.full((V,), -math.inf),
            torch.where(torch.rand(V, generator=g) < 1e-3, n, -math.inf), torch.where(torch.arange(V) == V - 1, 1.0, -math.inf),
            torch.where(torch.arange(V) % 9 == 0, 5.0, n), torch.where(n > 2, math.inf, n), torch.full((V,), torch.finfo(torch.float32).min),
            torch.where(torch.rand(V, generator=g) < 0.5, -0.0, 0.0), n * 1e-42, n.sort().values, torch.where(torch.arange(V) < 300, n + 50, n)]
    z = torch.stack(rows)
    for K in (1, 17, 128):
        check_top(L, z, K)
        check_top(L, z[-3:], K)


@pytest.mark.parametrize("M,V,K", [(450, 33001, 20), (600, 40000, 1), (700, 5003, 40), (900, 5003, 128), (1300, 2500, 9)])
def test_top_logits_of_many_rows(L, M, V, K):
    """One and two rounds of rows over the device, three and four of them to an SM; every tenth row mostly equal or all -inf."""
    z = torch.randn(M, V, generator=torch.Generator().manual_seed(M))
    z[::20] = torch.round(z[::20])
    z[10::20] = -math.inf
    check_top(L, z, K)


def test_top_logits_with_nan(L):
    g = torch.Generator().manual_seed(1)
    z = torch.randn(6, 5003, generator=g)
    z[0, ::3] = math.nan
    z[1] = math.nan
    z[2, 40:] = math.nan
    z[3, :] = -math.inf
    z[3, 100:200] = math.nan
    z[4, 7] = math.nan
    for K in (1, 64, 128):
        check_top(L, z, K)
        check_top(L, z[:, :3000], K)

"""Calls of the LM head's losses at the edges of what they take: coefficients that are not finite, tokens listed twice, low
temperatures, lists that differ from row to row, products that gave up."""
import math

import pytest
import torch

from tests.test_gpu_headloss import draw, run

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def L():
    from paper_2512_15176_b200 import binding
    binding.lib()
    return binding


# One live row, rows whose G is held as two terms for both products, for dh alone, as one term.
ROWS = [1, 40, 100, 300]


def outside(x):
    return ~torch.isfinite(x.float())


@pytest.mark.parametrize("M", ROWS)
@pytest.mark.parametrize("K", [None, 5])
@pytest.mark.parametrize("where", ["weight", "grad"])
@pytest.mark.parametrize("value", [math.nan, math.inf, -math.inf])
def test_coefficients_that_are_not_finite_throughout(L, M, K, where, value):
    """Every entry of the formula's gradients is a sum with a term of inf or NaN in it."""
    h, w, ids, teacher, a, g = draw(M, M, 64, 150, K=K)
    (a if where == "weight" else g).fill_(value)
    loss, _, _, dh, dw = run(L, h, w, ids, teacher=teacher, weight=a, grad=g)
    assert outside(dh).all() and outside(dw).all()
    assert outside(loss).all() if where == "weight" else torch.isfinite(loss).all()


@pytest.mark.parametrize("M", ROWS[1:])
@pytest.mark.parametrize("value", [math.nan, math.inf])
@pytest.mark.parametrize("others", [0.0, 1.0])
def test_one_coefficient_that_is_not_finite(L, M, value, others):
    """Beside rows without an upstream gradient, and beside ordinary ones: their dh is the same as without that row."""
    h, w, ids, _, a, g = draw(M, M, 64, 150)
    g *= others
    row = M // 3
    keep = torch.arange(M) != row
    g[row] = 0.0
    want = run(L, h, w, ids, weight=a, grad=g)[3]
    g[row] = value
    _, _, _, dh, dw = run(L, h, w, ids, weight=a, grad=g)
    assert outside(dh[row]).all() and outside(dw).all()
    assert torch.isfinite(dh[keep].float()).all()
    # (a common scale of G is chosen anew: as much as its rounding to bf16 and dh's own, 2^-8 each of a row's largest terms)
    assert ((dh[keep].float() - want[keep].float()).abs() <= 2.0 ** -7 * w.float().abs().max() * a[keep].cuda()[:, None] * g[keep].abs().cuda()[:, None] * 2).all()


def test_rows_without_a_gradient_stay_at_zero(L):
    h, w, ids, _, a, _ = draw(2, 30, 64, 150)
    _, _, _, dh, dw = run(L, h, w, ids, weight=a, grad=torch.zeros(30))
    assert not dh.any() and not dw.any()


@pytest.mark.parametrize("M,K", [(5, 6), (40, 8), (40, 9), (200, 20), (150, 128)])
def test_the_divergence_of_lists_that_repeat_tokens(L, M, K):
    """The list's distribution over tokens: what stands twice counts by its sum, in the loss as in its gradients."""
    tau, V, hid = 1.5, 60, 64
    h, w, _, _, a, g = draw(M + K, M, hid, V)
    gen = torch.Generator().manual_seed(K)
    ids = torch.randint(V // 3, (M, K), generator=gen).int()
    teacher = 3 * torch.randn(M, K, generator=gen)
    ids[0] = 7                                                  # one token: the divergence of a sure teacher
    ids[1, K // 2:] = -1
    teacher[2, ::2] = -math.inf                                 # entries without probability, some of a token that has some
    teacher[3, 1:] = teacher[3, 0] - 300.0                      # and some whose probability is below fp32's least
    loss, _, _, dh, dw = run(L, h, w, ids, teacher=teacher, tau=tau, weight=a, grad=g)
    live = (ids >= 0).double()
    t = torch.softmax(torch.where(ids >= 0, teacher.double() / tau, -math.inf), 1) * live
    dense = torch.zeros(M, V, dtype=torch.float64).scatter_add_(1, ids.clamp_min(0).long(), t)
    logp = torch.log_softmax(h.double() @ w.double().T / tau, 1)
    each = torch.where(dense > 0, dense * (torch.log(torch.where(dense > 0, dense, 1.0)) - logp), 0.0).sum(1)
    want = a.double() * tau ** 2 * each
    # z by plain sums and lse: 2^-19 of the largest of them; a logarithm and an exponential of t each a few 2^-24 of |log t| <= 5
    tol = a.double() * tau ** 2 * (2.0 ** -19 * logp.abs().amax(1) + 2.0 ** -20)
    assert ((loss.cpu().double() - want).abs() <= tol).all(), ((loss.cpu().double() - want).abs() / tol).max()
    assert (loss.cpu() >= -tol).all()                           # a divergence is not negative


@pytest.mark.parametrize("tau", [2.0 ** -20, 1e-4, 3e-3])
@pytest.mark.parametrize("M,K", [(6, 4), (140, 12)])
@pytest.mark.parametrize("hid,sure", [(64, 8.0), (8192, 50.0)])
def test_low_temperatures(L, M, K, hid, sure, tau):
    """p and t are all but sure, the loss about tau times a difference of logits; z's rounding / tau is beyond the exponential's
    range at the lowest."""
    h, w, ids, teacher, a, _ = draw(M, M, hid, 90, K=K, sure=sure)
    loss, lse, _, dh, dw = run(L, h, w, ids, teacher=teacher, tau=tau, weight=a)
    tau = torch.tensor(tau).double()                            # as the call has it
    z = h.double() @ w.double().T
    logp, t = torch.log_softmax(z / tau, 1), torch.softmax(teacher.double() / tau, 1)
    want = a.double() * tau * tau * torch.where(t > 0, t * (torch.log(torch.where(t > 0, t, 1.0)) - torch.gather(logp, 1, ids.long())), 0.0).sum(1)
    # z off by (hid / 16 + 8) steps of the accumulator, lse's reference by 2^-24 of it, and 2^-20 for what is left of the sums
    dz = (hid / 16 + 8) * 2.0 ** -23 * (h.double().abs() @ w.double().abs().T).amax(1)
    tol = a.double() * tau * (2 * dz + 2.0 ** -20 * z.abs().amax(1) + 2.0 ** -20 * tau)
    assert ((loss.cpu().double() - want).abs() <= tol).all(), ((loss.cpu().double() - want).abs() / tol).max()
    assert torch.isfinite(lse).all() and torch.isfinite(dh.float()).all() and torch.isfinite(dw.float()).all()


def test_lists_that_differ_from_row_to_row(L):
    """No two neighbouring rows have their listed tokens in the same columns, or as many of them: nothing, one, or all of a
    chunk of 32.  Every row's z and lse against the formula, in tiles of the rows as they are (short lists) and of lists by id."""
    for M, K in ((64, 8), (96, 128), (300, 128), (300, 33)):
        hid, V = 128, 3000
        h, w, _, teacher, a, g = draw(M, M, hid, V, K=K)
        gen = torch.Generator().manual_seed(M + K)
        ids = torch.full((M, K), -1, dtype=torch.int32)
        for m in range(M):
            n = 1 + (m * 37) % K
            if m % 4 == 0:
                pick = torch.randperm(V, generator=gen)[:n]
            elif m % 4 == 1:
                pick = (32 * (m % 90) + torch.arange(n)) % V    # a chunk, and what is behind it
            elif m % 4 == 2:
                pick = V - 1 - torch.arange(n)
            else:
                pick = (torch.arange(n) * 32 + m % 32) % V      # one to a chunk
            ids[m, :n] = pick.int()
        loss, lse, tl, dh, dw = run(L, h, w, ids, teacher=teacher, weight=a, grad=g)
        z = h.double() @ w.double().T
        dz = (hid / 16 + 8) * 2.0 ** -23 * (h.double().abs() @ w.double().abs().T).amax(1)
        want = torch.logsumexp(z, 1)
        assert ((lse.cpu().double() - want).abs() <= dz + 2.0 ** -20 + 2.0 ** -21 * want.abs()).all()
        zt = torch.gather(z, 1, ids.clamp_min(0).long())
        err = (tl.cpu().double() - zt).abs()
        assert (err[ids >= 0] <= dz[:, None].expand(M, K)[ids >= 0]).all() and (tl.cpu()[ids < 0] == 0).all()
        t = torch.softmax(torch.where(ids >= 0, teacher.double(), -math.inf), 1)
        each = torch.where(ids >= 0, t * (torch.log(torch.where(t > 0, t, 1.0)) - zt + want[:, None]), 0.0).sum(1)
        tol = a.double() * (2 * dz + 2.0 ** -20 + 2.0 ** -20 * (want.abs() + z.abs().amax(1) + 20))
        assert ((loss.cpu().double() - a.double() * each).abs() <= tol).all()


@pytest.mark.parametrize("M,V", [(1, 40), (70, 513), (300, 1000), (600, 2049)])
def test_gradients_of_a_product_that_gave_up_are_nan(L, M, V):
    """Both gradients, each alone, and nothing behind their ends; the next call is right again."""
    hid = 192
    h, w, ids, _, a, g = draw(M, M, hid, V)
    want = run(L, h, w, ids, weight=a, grad=g)
    h_, w_, t_, a_, g_ = (x.cuda() for x in (h, w, ids.view(-1), a, g))
    ws = torch.empty(L.deer_lmhead_loss_workspace_bytes(M, hid, V, 1, True), dtype=torch.uint8, device="cuda")
    room_h, room_w = (torch.full((n * hid + 64,), 3.0, dtype=torch.bfloat16, device="cuda") for n in (M, V))
    dh, dw = room_h[:M * hid], room_w[:V * hid]

    def grad(dh, dw):
        L.deer_lmhead_loss_grad(h_, w_, t_, want[1], want[2], dh, dw, ws, a_, g_)

    for dh_, dw_ in ((dh, dw), (None, dw), (dh, None)):
        grad(dh_, dw_)
        for x, y in ((dh_, want[3]), (dw_, want[4])):
            assert x is None or torch.equal(x.view_as(y), y)
        L.deer_selftest_lmhead_gave_up(h_, w_, 1, dh_, dw_, ws)
        for x in (dh_, dw_):
            assert x is None or torch.isnan(x).all()
    ws.fill_(0x7f)                                              # (no call has left this: places and counts far out of range)
    dh.fill_(0.0)
    L.deer_selftest_lmhead_gave_up(h_, w_, 1, dh, dw, ws)
    assert torch.isnan(dh).all() and torch.isnan(dw).all()
    assert (room_h[M * hid:] == 3).all() and (room_w[V * hid:] == 3).all()
    grad(dh, dw)
    assert torch.equal(dh.view_as(want[3]), want[3]) and torch.equal(dw.view_as(want[4]), want[4])

"""Pins of the oracle's LM-head losses: torch's cross entropy, KL divergence and autograd in 64 bits, central differences,
row weights, repeated and ended lists; top logits against a stable sort."""
import numpy as np
import pytest
import torch

from oracle import deer_oracle as O


def _draw(seed, M, hid, V, K):
    rng = np.random.default_rng(seed)
    ids = np.stack([rng.permutation(V)[:K] for _ in range(M)]).astype(np.int32)
    return (rng.standard_normal((M, hid)), rng.standard_normal((V, hid)) / np.sqrt(hid), ids, 2 * rng.standard_normal((M, K)),
            rng.uniform(0.5, 2.0, M), rng.uniform(-1.0, 2.0, M))


def test_cross_entropy_is_torchs():
    h, w, ids, _, a, g = _draw(1, 7, 12, 31, 1)
    ids[2] = -1
    th, tw = torch.tensor(h, requires_grad=True), torch.tensor(w, requires_grad=True)
    each = torch.nn.functional.cross_entropy(th @ tw.T, torch.tensor(ids[:, 0]).long(), ignore_index=-1, reduction="none") * torch.tensor(a)
    (each * torch.tensor(g)).sum().backward()
    loss, lse, *_ = O.head_loss(h, w, ids, row_weight=a)
    np.testing.assert_allclose(loss, each.detach().numpy(), rtol=1e-12, atol=1e-13)
    np.testing.assert_allclose(lse, np.where(ids[:, 0] < 0, 0, torch.logsumexp(th @ tw.T, 1).detach().numpy()), rtol=1e-12)
    dh, dw, _ = O.head_loss_grad(h, w, ids, row_weight=a, grad_loss=g)
    np.testing.assert_allclose(dh, th.grad.numpy(), rtol=1e-10, atol=1e-13)
    np.testing.assert_allclose(dw, tw.grad.numpy(), rtol=1e-10, atol=1e-13)


@pytest.mark.parametrize("tau", [0.7, 1.0, 2.0])
def test_distillation_is_the_divergence(tau):
    M, K, V = 6, 5, 23
    h, w, ids, teacher, a, g = _draw(2, M, 9, V, K)
    ids[1, 3:] = -1
    teacher[4, 2] = -np.inf
    full = np.full((M, V), -np.inf)                           # the teacher's row with everything unlisted at -inf
    for m in range(M):
        for j in range(K if m != 1 else 3):
            full[m, ids[m, j]] = teacher[m, j]
    th, tw = torch.tensor(h, requires_grad=True), torch.tensor(w, requires_grad=True)
    t = torch.softmax(torch.tensor(full) / tau, 1)
    logp = torch.log_softmax(th @ tw.T / tau, 1)
    each = torch.where(t > 0, t * (torch.log(torch.where(t > 0, t, 1.0)) - logp), 0.0).sum(1) * tau ** 2 * torch.tensor(a)
    (each * torch.tensor(g)).sum().backward()
    loss, *_ = O.head_loss(h, w, ids, teacher, tau, a)
    np.testing.assert_allclose(loss, each.detach().numpy(), rtol=1e-11, atol=1e-13)
    dh, dw, _ = O.head_loss_grad(h, w, ids, teacher, tau, a, g)
    np.testing.assert_allclose(dh, th.grad.numpy(), rtol=1e-10, atol=1e-13)
    np.testing.assert_allclose(dw, tw.grad.numpy(), rtol=1e-10, atol=1e-13)


def test_gradients_against_differences():
    h, w, ids, teacher, a, g = _draw(3, 4, 6, 11, 3)
    ids[0, 1] = ids[0, 0]                                     # a token listed twice
    ids[3] = -1
    total = lambda h_, w_: (g * O.head_loss(h_, w_, ids, teacher, 1.3, a)[0]).sum()  # noqa: E731
    dh, dw, _ = O.head_loss_grad(h, w, ids, teacher, 1.3, a, g)
    for x, dx in ((h, dh), (w, dw)):
        for at in np.ndindex(x.shape):
            keep, e = x[at], 1e-5
            x[at] = keep + e
            up = total(h, w)
            x[at] = keep - e
            down = total(h, w)
            x[at] = keep
            assert abs((up - down) / (2 * e) - dx[at]) < 1e-8


def test_rows_without_part():
    h, w, ids, teacher, a, g = _draw(4, 5, 8, 13, 4)
    ids[0, 0], a[1], teacher[2] = -1, 0.0, -np.inf
    h[0] = np.nan
    h[1] = 1.0
    loss, lse, *_ = O.head_loss(np.nan_to_num(h), w, ids, teacher, 1.0, a)
    assert (loss[:3] == 0).all() and (loss[3:] != 0).all() and (lse[:2] == 0).all()
    dh, dw, G = O.head_loss_grad(np.nan_to_num(h), w, ids, teacher, 1.0, a, g)
    assert (dh[:3] == 0).all() and (G[:3] == 0).all() and np.isfinite(dw).all()
    # the other rows alone give the same
    alone = O.head_loss_grad(h[3:], w, ids[3:], teacher[3:], 1.0, a[3:], g[3:])
    np.testing.assert_allclose(dw, alone[1], rtol=1e-12, atol=1e-14)


def test_top_logits_is_a_stable_sort():
    rng = np.random.default_rng(5)
    z = rng.integers(-4, 5, (6, 40)).astype(np.float32)      # ties everywhere
    z[1, 3], z[1, 7], z[2] = np.inf, -np.inf, 0.0
    z[2, ::2] = -0.0
    ids, values = O.top_logits(z, 9)
    want = torch.sort(torch.tensor(z) + 0.0, dim=1, descending=True, stable=True)
    np.testing.assert_array_equal(ids, want.indices[:, :9].numpy())
    np.testing.assert_array_equal(values, np.take_along_axis(z, ids.astype(np.int64), 1))
    z[3, 5] = np.nan
    ids, values = O.top_logits(z[3:4, :7], 9)
    assert ids[0, 6] == 5 and np.isnan(values[0, 6]) and (ids[0, 7:] == -1).all() and (values[0, 7:] == -np.inf).all()


def test_targets_of_the_two_stages():
    from paper_2512_15176_b200.runner import distill_targets, refine_targets
    rng = np.random.default_rng(6)
    B, T, hid, V = 3, 10, 7, 19
    tokens, masked = torch.tensor(rng.integers(0, V, (B, T))), torch.tensor(rng.random((B, T)) < 0.6)
    t, R, alpha = torch.tensor([0.25, 0.5, 1.0]), torch.tensor([1, 4, 10]), 1.01
    h, w = rng.standard_normal((B * T, hid)), rng.standard_normal((V, hid))
    z = (h @ w.T).reshape(B, T, V)
    nll = np.log(np.exp(z).sum(2)) - np.take_along_axis(z, tokens.numpy()[:, :, None], 2)[:, :, 0]
    targets, weight = distill_targets(tokens, masked, t)
    assert targets.dtype == torch.int32 and targets.is_contiguous()
    loss = O.head_loss(h, w, targets.numpy()[:, None], row_weight=weight.numpy().astype(np.float64))[0].reshape(B, T)
    want = sum(nll[b, i] / float(t[b]) for b in range(B) for i in range(T) if masked[b, i])
    np.testing.assert_allclose(loss.sum(), want, rtol=1e-12)
    targets, weight = refine_targets(tokens, masked, R, alpha)
    loss = O.head_loss(h, w, targets.numpy()[:, None], row_weight=weight.numpy().astype(np.float64))[0].reshape(B, T)
    want = 0.0
    for b in range(B):
        for i in range(1, int(R[b]) + 1):
            at = T - int(R[b]) + i - 1
            if masked[b, at]:
                want += alpha ** (int(R[b]) - i) * nll[b, at]
    np.testing.assert_allclose(loss.sum(), want, rtol=1e-6)                    # (weights in fp32)

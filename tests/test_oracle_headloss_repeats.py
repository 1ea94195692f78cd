"""Pin of the oracle's divergence where a list names a token more than once: that of the distribution over tokens."""
import numpy as np
import torch

from oracle import deer_oracle as O


def test_a_token_listed_twice_is_one_token():
    rng = np.random.default_rng(7)
    M, K, hid, V, tau = 8, 6, 9, 5, 1.5
    h, w = rng.standard_normal((M, hid)), rng.standard_normal((V, hid))
    ids, teacher, a = rng.integers(0, V, (M, K)).astype(np.int32), 2 * rng.standard_normal((M, K)), rng.uniform(0.5, 2.0, M)
    ids[0], ids[1, 3:] = 2, -1
    teacher[2, ::2] = -np.inf
    loss = O.head_loss(h, w, ids, teacher, tau, a)[0]
    u = torch.where(torch.tensor(ids) >= 0, torch.tensor(teacher) / tau, -torch.inf)
    dense = torch.zeros(M, V, dtype=torch.float64).scatter_add_(1, torch.tensor(ids).clamp_min(0).long(), torch.softmax(u, 1))
    each = torch.nn.functional.kl_div(torch.log_softmax(torch.tensor(h @ w.T) / tau, 1), dense, reduction="none").sum(1)
    np.testing.assert_allclose(loss, (each * tau ** 2).numpy() * a, rtol=1e-11, atol=1e-13)
    assert (loss >= 0).all()
    # one token, six times: the cross entropy of that token
    sure = O.head_loss(h[:1] / tau, w, ids[:1, :1], row_weight=a[:1] * tau ** 2)[0]
    np.testing.assert_allclose(loss[:1], sure, rtol=1e-11)

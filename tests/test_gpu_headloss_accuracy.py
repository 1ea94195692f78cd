"""How near lse, the listed logits and the loss are, where worst-case bounds say little: means and root mean squares over rows
against 64 bits.  u = 2^-24, half a step of fp32; a step of the tensor cores' accumulation is 16 of hid.

Their accumulation rounds towards zero.  The mean of it where products' signs mix, 1.5e-8 of z a step, is given back: half of that
is the bound on what is left on average (without it, or with its sign wrong, twice or four times as much is)."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


@pytest.fixture(scope="module")
def HeadLoss():
    from paper_2512_15176_b200 import binding
    binding.lib()
    from paper_2512_15176_b200.runner import HeadLoss
    return HeadLoss


def inputs(kind, M, hid, V=2048):
    g = torch.Generator(device="cuda")
    g.manual_seed(hid + M)
    n = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
    w, h, best = n(V, hid) / math.sqrt(hid), n(M, hid), torch.randint(V, (M,), generator=g, device="cuda")
    if kind == "mixed":                        # logits of size 6, the largest of them about 20
        h = 6 * h
    elif kind == "sure":                       # one token's logit is 40
        row = w[best].bfloat16().float()
        h = h + 40 * row / row.square().sum(1, keepdim=True)
    else:                                      # all products positive
        w, h = w.abs(), 0.5 * h.abs()
    h, w = h.bfloat16(), w.bfloat16()
    return h, w, best, h.double() @ w.double().T


SIZES = [(M, hid) for M in (100, 600) for hid in (2048, 8192, 16384)]


@pytest.mark.parametrize("M,hid", SIZES)
def test_logits_of_either_sign(HeadLoss, M, hid):
    h, w, best, z = inputs("mixed", M, hid)
    head = HeadLoss(w, M, grad=False)
    head.cross_entropy(h, best.int())
    want = torch.logsumexp(z, 1)
    err = (head.lse.double() - want) / want
    steps = hid / 16
    left = 0.75e-8 * steps + 2 * U             # the mean, and lse's own rounding
    assert abs(err.mean().item()) <= left
    # around it: a rounding of up to 2u of the sum so far at each step, independent of one another
    assert err.square().mean().sqrt().item() <= left + 2 * U * math.sqrt(steps)
    # listed logits: 64 sums of hid / 64 terms side by side, whose roundings add up as hid / 64 steps' do, and their joining
    zt = z.gather(1, best[:, None])[:, 0]
    rms = (head.target_logit.double().view(-1) - zt).square().mean().sqrt() / zt.square().mean().sqrt()
    assert rms.item() <= U * (2 + math.sqrt(hid / 64)), rms.item() / U


@pytest.mark.parametrize("M,hid", SIZES)
def test_losses_of_sure_rows(HeadLoss, M, hid):
    """p is all but 1: lse and the target's z, 40 and its roundings, cancel.  What is left is the exponential's and logarithm's."""
    h, w, best, z = inputs("sure", M, hid)
    head = HeadLoss(w, M, grad=False)
    loss = head.cross_entropy(h, best.int())
    want = torch.logsumexp(z, 1) - z.gather(1, best[:, None])[:, 0]
    assert want.max() < 1e-6
    assert ((loss.double() - want).abs() <= 2.0 ** -20).all(), (loss.double() - want).abs().max()


@pytest.mark.parametrize("M,hid", SIZES + [(100, 65536)])
@pytest.mark.parametrize("kind", ["sure", "positive"])
def test_lse_of_unlisted_tokens(HeadLoss, M, hid, kind):
    """The accuracy that the header gives for lse: 1e-8 of the largest logit a step, 1e-7 where all products have one sign."""
    h, w, best, z = inputs(kind, M, hid)
    head = HeadLoss(w, M, grad=False)
    head.cross_entropy(h, ((best + 1) % w.shape[0]).int())
    want = torch.logsumexp(z, 1)
    bound = (1e-8 if kind == "sure" else 1e-7) * hid / 16 * z.amax(1) + 2.0 ** -20 + 8 * U * want.abs()
    err = (head.lse.double() - want).abs()
    assert err.mean() <= bound.mean(), (err / bound).max()

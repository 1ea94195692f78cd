"""The LM head's losses as a program uses them: behind a verify step, on streams, in graphs, with shared workspaces, with the
largest and the most padded batches; gradients against differences."""
import math

import numpy as np
import pytest
import torch

from oracle import deer_oracle as O
from tests.test_gpu_headloss import B, U, check, draw, f64

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def L():
    from paper_2512_15176_b200 import binding
    binding.lib()
    return binding


def bits(*tensors):
    return [t.clone() for t in tensors]


def same(a, b):
    return all(torch.equal(x.view(torch.uint8), y.view(torch.uint8)) for x, y in zip(a, b))


def step(head, h, ids, teacher, a, g):
    loss = head.distill(h, ids, teacher, 1.5, a) if teacher is not None else head.cross_entropy(h, ids[:, 0].contiguous(), a)
    dh, dw = head.backward(g)
    return bits(loss, head.lse, head.target_logit, dh, dw)


def on_gpu(*tensors):
    return [None if t is None else t.cuda() for t in tensors]


def test_from_a_verify_step_to_the_drafters_gradients(L):
    """Logits of the verifier's head -> its top logits -> the drafter's loss against them -> gradients."""
    from paper_2512_15176_b200.runner import HeadLoss
    M, hid_v, hid, V, K = 40, 256, 128, 2000, 16
    g = torch.Generator().manual_seed(2)
    hv, wv = torch.randn(M, hid_v, generator=g).bfloat16(), (0.3 * torch.randn(V, hid_v, generator=g)).bfloat16()
    logits, out = torch.empty(M, V, device="cuda"), torch.empty(M, dtype=torch.int32, device="cuda")
    ws = torch.empty(L.deer_lmhead_workspace_bytes(M, hid_v, V), dtype=torch.uint8, device="cuda")
    L.deer_lmhead_select(hv.cuda(), wv.cuda(), L.DEER_SEL_ARGMAX, 1.0, None, out, None, None, None, logits, ws)
    ids, teacher = torch.empty(M, K, dtype=torch.int32, device="cuda"), torch.empty(M, K, device="cuda")
    L.deer_top_logits(logits, ids, teacher)
    want_ids, want = O.top_logits(logits.cpu().numpy(), K)
    np.testing.assert_array_equal(ids.cpu().numpy(), want_ids)
    np.testing.assert_array_equal(teacher.cpu().numpy(), want)
    assert torch.equal(ids[:, 0], out)                                     # the argmax leads
    h, w, _, _, a, gl = draw(11, M, hid, V)
    head = HeadLoss(w.cuda(), M, top=K)
    got = step(head, h.cuda(), ids, teacher, a.cuda(), gl.cuda())
    torch.cuda.synchronize()
    check(got, h, w, ids, teacher, 1.5, a, gl)
    frozen_dh, none = head.backward(gl.cuda(), head=False)
    assert none is None and torch.equal(frozen_dh, got[3])


def test_verify_step_as_a_teacher(L):
    from paper_2512_15176_b200 import workload as W
    from paper_2512_15176_b200.runner import VerifyStep
    cfg = W.StepConfig("teacher", 2, 8, 2, 64, 8, 256, 2048, (40, 60), mode="sample", temperature=1.0, seed=31)
    lengths = W.seq_lengths(cfg)
    lay = W.kv_layout(cfg, lengths)
    kp, vp = W.kv_pools(cfg, lay.num_pages, sigma=1.0)
    vs = VerifyStep(cfg, L.KVCache.from_layout(lay, kp, vp), W.lm_head(cfg).cuda(), int(lengths.max()))
    vs.load(*W.block_qkv(cfg), W.hidden(cfg))
    vs.lmhead()
    ids, values = torch.empty(cfg.M, 8, dtype=torch.int32, device="cuda"), torch.empty(cfg.M, 8, device="cuda")
    vs.top_logits(ids, values)
    best = torch.topk(vs.logits, 8, dim=1)
    assert torch.equal(values, best.values) and torch.equal(ids[:, 0], vs.target_ids.view(-1))


@pytest.mark.parametrize("K", [None, 12])
def test_a_captured_step_follows_its_inputs(L, K):
    from paper_2512_15176_b200.runner import HeadLoss
    M, hid, V = 150, 128, 1500
    a_, b_ = draw(1, M, hid, V, K=K, live=0.9), draw(2, M, hid, V, K=K, live=0.3)
    now = [None if t is None else t.cuda() for t in a_]
    head = HeadLoss(now[1], M, top=K or 1)
    one = HeadLoss(now[1], M, top=K or 1)
    ids = now[2]

    def run(head):
        h, _, _, teacher, wt, g = now
        if K:
            loss = head.distill(h, ids, teacher, 1.5, wt)
        else:
            loss = head.cross_entropy(h, ids.view(-1), wt)
        return (loss, *head.backward(g))

    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        run(head)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=s):
            outs = run(head)
    torch.cuda.synchronize()
    for inputs in (a_, b_, a_):
        for dst, src in zip(now, inputs):
            if dst is not None:
                dst.copy_(src)
        for t in outs:
            t.fill_(9.0)
        graph.replay()
        torch.cuda.synchronize()
        got = bits(*outs)
        assert same(got, bits(*run(one)))
        check((outs[0], one.lse, one.target_logit, outs[1], outs[2]), *inputs[:4], *((1.5,) if K else (1.0,)), inputs[4], inputs[5])


def test_two_graphs_share_a_workspace(L):
    """Two captured steps of different sizes over one workspace, replayed in turn."""
    M, hid, V = 90, 128, 1200
    parts = []
    need = max(L.deer_lmhead_loss_workspace_bytes(m, hid, V, 1, g) for m in (M, 3 * M) for g in (False, True))
    ws = torch.empty(need, dtype=torch.uint8, device="cuda")
    s = torch.cuda.Stream()
    for i, m in enumerate((M, 3 * M)):
        h, w, ids, _, a, g = draw(40 + i, m, hid, V, live=0.7)
        h_, w_, ids_, a_, g_ = on_gpu(h, w, ids[:, 0].contiguous(), a, g)
        o = lambda *sh, dtype=torch.float32: torch.zeros(*sh, dtype=dtype, device="cuda")  # noqa: E731
        out = [o(m), o(m), o(m, 1), o(m, hid, dtype=torch.bfloat16), o(V, hid, dtype=torch.bfloat16)]

        def run():
            L.deer_lmhead_loss(h_, w_, ids_, out[0], out[1], out[2], ws, a_)
            L.deer_lmhead_loss_grad(h_, w_, ids_, out[1], out[2], out[3], out[4], ws, a_, g_)

        with torch.cuda.stream(s):
            run()
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph, stream=s):
                run()
        parts.append((graph, out, (h, w, ids, None, 1.0, a, g), (h_, w_, ids_, a_, g_)))
    for _ in range(2):
        for graph, out, _, _ in parts:
            for t in out:
                t.zero_()
        torch.cuda.synchronize()
        for graph, *_ in parts:
            graph.replay()
        torch.cuda.synchronize()
        for _, out, inputs, _ in parts:
            check(out, *inputs)


def test_two_streams_at_once(L):
    from paper_2512_15176_b200.runner import HeadLoss
    cases = [draw(60 + i, 200 + 70 * i, 256, 6000, K=K, live=0.8) for i, K in enumerate((None, 9))]
    heads, ins, alone = [], [], []
    for c in cases:
        x = on_gpu(*c)
        head = HeadLoss(x[1], x[0].shape[0], top=x[2].shape[1])
        heads.append(head)
        ins.append((x[0], x[2], x[3], x[4], x[5]))
        alone.append(step(head, *ins[-1]))
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in cases]
    for _ in range(5):
        got = []
        for s, head, x in zip(streams, heads, ins):
            with torch.cuda.stream(s):
                got.append(step(head, *x))
        torch.cuda.synchronize()
        for a, b in zip(alone, got):
            assert same(a, b)


def test_explicit_stream(L):
    h, w, ids, _, a, g = draw(70, 50, 128, 700)
    h_, w_, t_, a_ = on_gpu(h, w, ids[:, 0].contiguous(), a)
    loss, lse, tl = (torch.zeros(50, device="cuda") for _ in range(3))
    ws = torch.empty(L.deer_lmhead_loss_workspace_bytes(50, 128, 700), dtype=torch.uint8, device="cuda")
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    L.deer_lmhead_loss(h_, w_, t_, loss, lse, tl, ws, a_, stream=s)
    s.synchronize()
    want = O.head_loss(f64(h), f64(w), ids.numpy(), row_weight=f64(a))[0]
    assert np.abs(f64(loss) - want).max() < 1e-4


def test_an_empty_batch(L):
    w = torch.randn(300, 128).bfloat16().cuda()
    e = lambda *s, dtype=torch.float32: torch.empty(*s, dtype=dtype, device="cuda")  # noqa: E731
    h, t, ws = e(0, 128, dtype=torch.bfloat16), e(0, dtype=torch.int32), e(16, dtype=torch.uint8)
    dw = torch.ones_like(w)
    L.deer_lmhead_loss(h, w, t, e(0), e(0), e(0), ws)
    L.deer_lmhead_loss_grad(h, w, t, e(0), e(0), None, dw, ws)
    L.deer_top_logits(e(0, 50), e(0, 4, dtype=torch.int32), e(0, 4))
    torch.cuda.synchronize()
    assert (dw == 0).all()


@pytest.mark.parametrize("M,K", [(2047, None), (2049, 5), (4500, None), (20000, 3)])
def test_many_rows_few_of_them_live(L, M, K):
    """The live rows' losses and the gradients are those of the live rows alone.  (Against the formula, not bit by bit: lse goes
    by other tiles in a batch of other size, within its tolerance.)"""
    from paper_2512_15176_b200.runner import HeadLoss
    hid, V = 64, 300
    h, w, ids, teacher, a, g = draw(M, M, hid, V, K=K, live=0.02)
    ids[[0, M - 1]] = 7 if K is None else torch.arange(K, dtype=torch.int32)
    a[M // 2] = 0.0
    live = (ids[:, 0] >= 0) & (a != 0)
    h[~live] = math.nan
    got = step(HeadLoss(w.cuda(), M, top=K or 1), *on_gpu(h, ids, teacher, a, g))
    few = [None if t is None else t[live].contiguous() for t in (h, ids, teacher, a, g)]
    at = live.cuda()
    check([t[at] for t in got[:4]] + [got[4]], few[0], w, few[1], few[2], 1.5 if K else 1.0, few[3], few[4])
    for t in (got[0], got[1], got[3]):
        assert (t[~at] == 0).all()


def test_the_most_rows(L):
    M, hid, V = 1 << 18, 64, 200
    h = torch.randn(M, hid, device="cuda").bfloat16()
    w = (torch.randn(V, hid, device="cuda") / 8).bfloat16()
    t = torch.full((M,), -1, dtype=torch.int32, device="cuda")
    at = torch.tensor([0, 77, 131072, M - 1], device="cuda")
    t[at] = torch.tensor([5, 199, 0, 77], dtype=torch.int32, device="cuda")
    e = lambda *s, dtype=torch.float32: torch.empty(*s, dtype=dtype, device="cuda")  # noqa: E731
    loss, lse, tl, dh, dw = e(M), e(M), e(M), e(M, hid, dtype=torch.bfloat16), e(V, hid, dtype=torch.bfloat16)
    ws = e(max(L.deer_lmhead_loss_workspace_bytes(M, hid, V, 1, g) for g in (False, True)), dtype=torch.uint8)
    L.deer_lmhead_loss(h, w, t, loss, lse, tl, ws)
    L.deer_lmhead_loss_grad(h, w, t, lse, tl, dh, dw, ws)
    torch.cuda.synchronize()
    check([x[at] if x is not dw else x for x in (loss, lse, tl.view(-1, 1), dh, dw)], h[at], w, t[at].view(-1, 1))
    assert int((loss != 0).sum()) == 4 and int(dh.abs().sum(1).count_nonzero()) == 4


def test_behind_four_gigabytes(L):
    """w and dw beyond 2^32 bytes, logits beyond 2^32 bytes: tokens and rows at the far end."""
    V, hid, M = 1_050_001, 2112, 3
    w = torch.empty(V, hid, dtype=torch.bfloat16, device="cuda").normal_(0, 0.02)
    h = torch.randn(M, hid, device="cuda").bfloat16()
    t = torch.tensor([V - 1, 3, V - 2], dtype=torch.int32, device="cuda")
    from paper_2512_15176_b200.runner import HeadLoss
    head = HeadLoss(w, M)
    loss = head.cross_entropy(h, t)
    dh, dw = head.backward()
    z = torch.cat([h.double() @ w[i:i + 100_000].double().T for i in range(0, V, 100_000)], 1)
    want = torch.logsumexp(z, 1) - z.gather(1, t.long()[:, None])[:, 0]
    dz = (hid / 16 + 8) * 2 * U * 40
    assert ((loss - want).abs() <= 2 * dz + 2.0 ** -20 + 16 * U * 40).all()
    p = torch.softmax(z, 1)
    p[torch.arange(M), t.long()] -= 1
    for rows in (torch.arange(V - 300, V, device="cuda"), torch.arange(0, 300, device="cuda"), torch.arange(V // 2, V // 2 + 300, device="cuda")):
        ref = p[:, rows].T @ h.double()
        bound = B * ref.abs() + (p[:, rows].abs().T @ h.double().abs()) * (2 * dz + 2.0 ** -15) + 2.0 ** -133
        assert ((dw[rows].double() - ref).abs() <= bound).all()
    ref = torch.zeros(M, hid, dtype=torch.float64, device="cuda")
    for i in range(0, V, 100_000):
        ref += p[:, i:i + 100_000] @ w[i:i + 100_000].double()
    assert ((dh.double() - ref).norm() / ref.norm()).item() < B
    del w, dw, dh, z, p, head
    torch.cuda.empty_cache()
    rows, V = 9000, 151_937
    z = torch.empty(rows, V, device="cuda").normal_()
    ids, values = torch.empty(rows, 5, dtype=torch.int32, device="cuda"), torch.empty(rows, 5, device="cuda")
    L.deer_top_logits(z, ids, values)
    for r in (0, 7066, 7067, 7068, rows - 1):                              # 2^30 values lie before row 7067
        best = torch.topk(z[r], 5)
        assert torch.equal(values[r], best.values) and torch.equal(ids[r].long(), best.indices)


@pytest.mark.parametrize("K", [None, 6])
def test_gradients_against_differences(L, K):
    """One coordinate moved by an exact step e both ways.  The losses are off by their tolerance, the difference by its third
    order, e^3 / 3 of |f'''| <= r^3 with r the coordinate's range over the vocabulary (dh) or of h (dw)."""
    from paper_2512_15176_b200.runner import HeadLoss
    M, hid, V, e = 6, 64, 90, 2.0 ** -4
    g = torch.Generator().manual_seed(4)
    h = (torch.randint(-24, 25, (M, hid), generator=g).float() / 16).bfloat16()          # with room for +-1/16
    w = (torch.randint(-24, 25, (V, hid), generator=g).float() / 128).bfloat16()
    _, _, ids, teacher, a, gl = draw(14, M, hid, V, K=K)
    gl = torch.ones(M)

    def loss(h, w):
        head = HeadLoss(w.cuda(), M, top=K or 1)
        out = head.distill(h.cuda(), ids.cuda(), teacher.cuda(), 1.5, a.cuda()) if K else head.cross_entropy(h.cuda(), ids.cuda().view(-1), a.cuda())
        return out.double().sum().item(), head

    _, head = loss(h, w)
    dh, dw = (f64(t) for t in head.backward(gl.cuda()))
    tau = 1.5 if K else 1.0
    noise = float((tau ** 2 * a).sum()) * (2 * (hid / 16 + 8) * 2 * U * 12 + 2.0 ** -19 + 32 * U * 10)
    for k in range(24):
        c = int(torch.randint(hid, (1,), generator=g))
        for x, grad, r in ((h, dh, k % M), (w, dw, int(ids[k % M, 0]) if k % 2 else k)):
            step_ = e if x is h else e / 8
            up, down = x.clone(), x.clone()
            up[r, c] += step_
            down[r, c] -= step_
            assert up[r, c] - x[r, c] == step_ and x[r, c] - down[r, c] == step_
            diff = loss(*((up, w) if x is h else (h, up)))[0] - loss(*((down, w) if x is h else (h, down)))[0]
            span = (2 * w.abs().max() if x is h else h.abs().max()).item() / tau
            third = step_ ** 3 / 3 * span ** 3 * float((tau ** 2 * a).sum())
            assert abs(diff - 2 * step_ * grad[r, c]) <= 2 * noise + third + 2 * step_ * (2 * B * abs(grad[r, c]) + 1e-6), (k, r, c)


def test_autograd_carries_on_from_dh(L):
    """The drafter's own graph takes dh: a small trunk's weights get the gradient of the whole."""
    from paper_2512_15176_b200.runner import HeadLoss
    M, hid, V = 24, 64, 200
    h, w, ids, _, a, _ = draw(15, M, hid, V)
    trunk = torch.nn.Linear(hid, hid, bias=False, dtype=torch.bfloat16, device="cuda")
    x = h.cuda()
    y = trunk(x)
    head = HeadLoss(w.cuda(), M)
    head.cross_entropy(y.detach(), ids.cuda().view(-1), a.cuda())
    dh, dw = head.backward(torch.full((M,), 1.0 / M, device="cuda"))
    y.backward(dh)
    ref_trunk = trunk.weight.detach().double().requires_grad_()
    yd = x.double() @ ref_trunk.T
    each = torch.nn.functional.cross_entropy(yd @ w.cuda().double().T, ids.cuda().view(-1).long(), reduction="none")
    (each * a.cuda().double()).mean().backward()
    rel = ((trunk.weight.grad.double() - ref_trunk.grad).norm() / ref_trunk.grad.norm()).item()
    # roundings on the way: y, dh, and the trunk's own product, half a bf16 step each; y's also enters p
    assert rel < 8 * B, rel


def test_refused_on_other_devices_sizes_and_orders(L):
    from paper_2512_15176_b200.runner import HeadLoss
    w = torch.zeros(300, 128, dtype=torch.bfloat16, device="cuda")
    head = HeadLoss(w, 5, top=3)
    h, ids, teacher = torch.zeros(5, 128, dtype=torch.bfloat16, device="cuda"), torch.zeros(5, 3, dtype=torch.int32, device="cuda"), torch.zeros(5, 3, device="cuda")
    with pytest.raises(AssertionError, match="follows a loss"):
        head.backward()
    head.distill(h, ids, teacher)
    for bad in (dict(h=h.cpu()), dict(h=h[:4]), dict(h=h.float()), dict(ids=ids[:, :2]), dict(ids=ids.long()), dict(teacher=teacher[:, :2]), dict(ids=ids.cpu())):
        with pytest.raises(L.DeerError):
            head.distill(**{**dict(h=h, ids=ids, teacher=teacher), **bad})
    with pytest.raises(L.DeerError):
        head.backward(torch.zeros(4, device="cuda"))
    with pytest.raises(AssertionError, match="contiguous"):
        head.distill(torch.zeros(128, 5, dtype=torch.bfloat16, device="cuda").t(), ids, teacher)
    with pytest.raises(L.DeerError):
        L.HeadLossBuffers(w.float(), 5)
    with pytest.raises(L.DeerError):
        HeadLoss(w, 5, grad=False).buffers.run_grad(h, ids[:, 0].contiguous())
    torch.cuda.synchronize()

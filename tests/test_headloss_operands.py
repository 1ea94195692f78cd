"""What the LM-head losses and the top logits refuse: sizes, pointers and workspaces in the library, operands of another type,
size or device in the binding.  No kernel runs here."""
import pytest
import torch

BF, F32, I32 = torch.bfloat16, torch.float32, torch.int32
FAKE = 0x1000          # never dereferenced on the host


@pytest.fixture(scope="module")
def L():
    from paper_2512_15176_b200 import build
    build.build()
    from paper_2512_15176_b200 import binding
    binding.lib()
    return binding


def z(*shape, dtype=BF):
    return torch.zeros(*shape, dtype=dtype)


def test_library_refusals(L):
    lib = L.lib()

    def loss(h=FAKE, w=FAKE, ids=FAKE, weight=None, M=5, hid=128, V=300, out=FAKE, ws=FAKE, size=1 << 30):
        return lib.deer_lmhead_loss(h, w, ids, weight, M, hid, V, out, out, out, ws, size, None)

    def grad(K=4, tau=1.0, teacher=FAKE, lse=FAKE, dh=2 * FAKE, dw=2 * FAKE, M=5, hid=128, V=300, ws=FAKE, size=1 << 30):
        return lib.deer_lmhead_distill_grad(FAKE, FAKE, FAKE, teacher, K, tau, None, None, lse, FAKE, M, hid, V, dh, dw, ws, size, None)

    bad, no = L.DEER_ERR_INVALID_ARG, L.DEER_ERR_UNSUPPORTED
    assert loss(h=None) == loss(w=None) == loss(ids=None) == loss(out=None) == bad
    assert loss(h=FAKE + 8) == loss(w=FAKE + 2) == loss(ids=FAKE + 1) == loss(weight=FAKE + 2) == loss(out=FAKE + 3) == bad
    assert loss(M=-1) == loss(V=0) == bad
    assert loss(hid=96) == loss(hid=0) == loss(hid=65536 + 64) == loss(M=(1 << 18) + 1) == no
    need = L.deer_lmhead_loss_workspace_bytes(5, 128, 300)
    assert 0 < need < 1 << 20
    assert loss(ws=None) == loss(ws=FAKE + 4) == loss(size=need - 1) == L.DEER_ERR_WORKSPACE
    assert loss(M=0, ws=None, size=0) == L.DEER_OK                     # an empty batch has no losses
    assert grad(K=0) == grad(K=129) == no
    assert grad(tau=0.0) == grad(tau=-1.0) == grad(tau=float("nan")) == grad(tau=float("inf")) == bad
    assert grad(teacher=None) == grad(lse=None) == grad(dh=None, dw=None) == grad(dh=FAKE + 8) == grad(dw=FAKE + 4) == bad
    assert grad(dh=FAKE) == grad(dw=FAKE) == bad                       # in the operand's place
    assert grad(size=L.deer_lmhead_loss_workspace_bytes(5, 128, 300, 4, True) - 1) == L.DEER_ERR_WORKSPACE
    assert grad(M=0, dw=None, ws=None, size=0) == L.DEER_OK
    top = lambda M=2, V=300, x=FAKE, K=8, i=FAKE, v=FAKE: lib.deer_top_logits(M, V, x, K, i, v, None)  # noqa: E731
    assert top(M=-1) == top(V=0) == top(x=None) == top(x=FAKE + 4) == top(i=None) == top(v=FAKE + 2) == bad
    assert top(K=0) == top(K=129) == top(M=(1 << 24) + 1) == no
    assert top(M=0) == L.DEER_OK


def test_workspace_grows_with_the_call(L):
    size = L.deer_lmhead_loss_workspace_bytes
    assert size(0, 128, 300) == size(5, 96, 300) == size(5, 128, 0) == size(5, 128, 300, 129) == 0
    # bounded by rows, not by rows x vocabulary: the logits are never kept
    assert size(4096, 2048, 151936) < 64 << 20 and size(4096, 2048, 151936, 1, True) < 600 << 20
    assert 4096 * 151936 * 4 > 2000 << 20


def _refused(L, call, good, bad):
    for name, values in bad.items():
        for v in values:
            with pytest.raises(L.DeerError) as e:
                call(**{**good, name: v})
            assert e.value.code == L.DEER_ERR_INVALID_ARG, (name, str(e.value))


def test_binding_refusals(L):
    f = lambda *s: z(*s, dtype=F32)  # noqa: E731
    i = lambda *s: z(*s, dtype=I32)  # noqa: E731
    ws = z(64, dtype=torch.uint8)
    one = dict(h=z(5, 128), w=z(300, 128), targets=i(5), lse=f(5), target_logit=f(5), workspace=ws, row_weight=f(5))
    some = dict(h=[z(5, 64), z(5, 128, dtype=F32), z(640)], w=[z(300, 64), z(300, 128, dtype=F32)], lse=[f(4), None], target_logit=[f(4), None],
                row_weight=[f(6), z(5)])
    _refused(L, L.deer_lmhead_loss, {**one, "loss": f(5)}, {**some, "targets": [i(4), z(5, dtype=torch.int64), None], "loss": [f(4), z(5), None]})
    _refused(L, L.deer_lmhead_loss_grad, {**one, "dh": z(5, 128), "dw": z(300, 128)},
             {**some, "dh": [z(4, 128), f(5, 128)], "dw": [z(299, 128), f(300, 128)], "grad_loss": [f(4), z(5)]})
    del one["targets"]
    some["target_logit"] = [f(5), f(4, 7)]
    lists = dict(ids=i(5, 7), teacher=f(5, 7), temperature=1.0, target_logit=f(5, 7))
    wrong = dict(ids=[i(5, 6), i(4, 7), z(5, 7, dtype=torch.int64), None], teacher=[f(5, 6), z(5, 7), None])
    _refused(L, L.deer_lmhead_distill, {**one, **lists, "loss": f(5)}, {**some, **wrong, "loss": [f(4)]})
    _refused(L, L.deer_lmhead_distill_grad, {**one, **lists, "dh": z(5, 128), "dw": None}, {**some, **wrong, "dh": [f(5, 128)]})
    _refused(L, L.deer_top_logits, dict(logits=f(2, 300), ids=i(2, 8), values=f(2, 8)),
             dict(logits=[z(2, 300), f(600)], ids=[i(2, 7), i(3, 8), f(2, 8)], values=[f(2, 7), z(2, 8)]))
    # right in everything but the device
    for call, good in ((L.deer_lmhead_loss, {**one, "targets": i(5), "loss": f(5)}), (L.deer_top_logits, dict(logits=f(2, 300), ids=i(2, 8), values=f(2, 8)))):
        with pytest.raises(L.DeerError, match="CUDA device"):
            call(**good)

"""More of what the LM-head losses refuse on the host.  No kernel runs here."""
import pytest
import torch

FAKE = 0x1000          # never dereferenced on the host


@pytest.fixture(scope="module")
def L():
    from paper_2512_15176_b200 import build
    build.build()
    from paper_2512_15176_b200 import binding
    binding.lib()
    return binding


def test_the_self_test_checks_its_operands(L):
    need = L.deer_lmhead_loss_workspace_bytes(5, 128, 300, 4, True)
    call = lambda M=5, hid=128, V=300, K=4, dh=FAKE, dw=FAKE, ws=FAKE, size=need: lib(M, hid, V, K, dh, dw, ws, size, None)  # noqa: E731
    lib = L.lib().deer_selftest_lmhead_gave_up
    assert call(M=0) == call(V=0) == call(dh=None, dw=None) == call(dh=FAKE + 8) == call(dw=FAKE + 2) == L.DEER_ERR_INVALID_ARG
    assert call(hid=96) == call(K=0) == call(K=129) == L.DEER_ERR_UNSUPPORTED
    assert call(ws=None) == call(ws=FAKE + 4) == call(size=need - 1) == L.DEER_ERR_WORKSPACE
    z = lambda *s: torch.zeros(*s, dtype=torch.bfloat16)  # noqa: E731
    for bad in (dict(dh=z(4, 128)), dict(dw=torch.zeros(300, 128)), dict(h=z(5, 64))):
        with pytest.raises(L.DeerError):
            L.deer_selftest_lmhead_gave_up(**{**dict(h=z(5, 128), w=z(300, 128), K=4, dh=z(5, 128), dw=z(300, 128), workspace=None), **bad})


def test_temperatures_that_z_has_no_bits_for(L):
    need = L.deer_lmhead_loss_workspace_bytes(5, 128, 300, 4, True)
    lib = L.lib()
    loss = lambda tau, size: lib.deer_lmhead_distill(FAKE, FAKE, FAKE, FAKE, 4, tau, None, 5, 128, 300, FAKE, FAKE, FAKE, FAKE, size, None)  # noqa: E731
    grad = lambda tau, size: lib.deer_lmhead_distill_grad(FAKE, FAKE, FAKE, FAKE, 4, tau, None, None, FAKE, FAKE, 5, 128, 300, 2 * FAKE, None,  # noqa: E731
                                                          FAKE, size, None)
    assert loss(9e-7, need) == grad(1e-39, need) == loss(1.1e6, need) == grad(1e30, need) == L.DEER_ERR_UNSUPPORTED
    assert loss(2.0 ** -20, 16) == grad(2.0 ** -20, 16) == loss(2.0 ** 20, 16) == L.DEER_ERR_WORKSPACE

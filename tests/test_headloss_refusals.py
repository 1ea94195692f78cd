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


def test_gradients_that_overlap_an_operand(L):
    M, hid, V, K = 5, 128, 300, 4
    need = L.deer_lmhead_loss_workspace_bytes(M, hid, V, K, True)
    place, at = {}, 0x100000
    for name, n in (("h", M * hid * 2), ("w", V * hid * 2), ("ids", M * K * 4), ("teacher", M * K * 4), ("weight", M * 4), ("grad", M * 4), ("lse", M * 4),
                    ("tl", M * K * 4), ("dh", M * hid * 2), ("dw", V * hid * 2), ("ws", need)):
        place[name] = (at, n)
        at += (n + 15) // 16 * 16

    def call(cross_entropy=False, size=need, **moved):
        p = {k: moved.get(k, v[0]) for k, v in place.items()}
        if cross_entropy:
            return L.lib().deer_lmhead_loss_grad(p["h"], p["w"], p["ids"], p["weight"], p["grad"], p["lse"], p["tl"], M, hid, V, p["dh"], p["dw"], p["ws"],
                                                 size, None)
        return L.lib().deer_lmhead_distill_grad(p["h"], p["w"], p["ids"], p["teacher"], K, 1.0, p["weight"], p["grad"], p["lse"], p["tl"], M, hid, V,
                                                p["dh"], p["dw"], p["ws"], size, None)

    for out, n in (("dh", M * hid * 2), ("dw", V * hid * 2)):
        for other, (start, size) in place.items():
            if other == out:
                continue
            # over its first and its last bytes
            for moved in (start + (size - 1) // 16 * 16, start - (n - 1) // 16 * 16, start):
                gone = {k: None for k in ("dh", "dw") if k not in (out, other)}
                assert call(**{out: moved}, **gone) == L.DEER_ERR_INVALID_ARG, (out, other)
                assert b"overlaps" in L.lib().deer_last_error()
            if other != "teacher":
                assert call(True, **{out: start}, **gone) == L.DEER_ERR_INVALID_ARG, (out, other)

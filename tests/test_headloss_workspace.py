"""What the LM-head losses' workspaces grow with: rows, and rows x tiles of the vocabulary.  No kernel runs here."""
import pytest


@pytest.fixture(scope="module")
def size():
    from paper_2512_15176_b200 import build
    build.build()
    from paper_2512_15176_b200 import binding
    binding.lib()
    return binding.deer_lmhead_loss_workspace_bytes


def padded(M):
    return (M + 255) // 256 * 256


@pytest.mark.parametrize("hid", [64, 2048])
@pytest.mark.parametrize("M", [1, 2049, 4096, 1 << 17, 1 << 18])
def test_loss_holds_seventeen_bytes_for_a_row_and_a_tile(size, M, hid):
    """Two partial sums of eight bytes and a list's place; tiles are 256 columns wide for many rows, 64 at least."""
    rows = padded(M)
    for K in (1, 128):
        fixed = rows * (2 * hid + 4 + 12 * K) + 4 * M + 10 * 1024
        before = size(M, hid, 10000, K)
        for V in (50257, 151936, 1 << 20):
            need = size(M, hid, V, K)
            assert 16 * rows * V / 256 <= need <= fixed + 17 * rows * (V / (64 if M < 4096 else 240) + 4)
            assert need > before
            before = need
        if K == 1 and M >= 4096:
            assert size(2 * M, hid, 151936) == 0 or abs(size(2 * M, hid, 151936) / size(M, hid, 151936) - 2) < 0.02
    # the logits of many rows are sixty times as much
    assert M < 4096 or size(M, hid, 151936) - 2 * rows * hid < rows * 151936 * 4 / 55


@pytest.mark.parametrize("M", [1, 4096, 1 << 17, 1 << 18])
def test_gradients_hold_a_piece_of_the_vocabulary(size, M):
    """G of 256 MB, or of 1024 columns where those are more; beside it the rows, partial dh and a byte for a row and a tile."""
    hid, rows = 64, padded(M)
    for V in (50257, 151936, 1 << 20):
        piece = max(256 << 20, rows * 1024 * 2)
        assert size(M, hid, V, 1, True) <= piece + rows * (2 * hid + 20 + V / 64 + 8) + max(rows, 148 * 256) * hid * 4 + (1 << 20)
    assert size(1 << 18, hid, 151936, 1, True) > (1 << 18) * 1024 * 2

"""How much memory the gradients of the vocabulary's loss ask for where the library chooses the pieces (CPU only): what lemo.h says."""
import pytest

from paper_2501_09767_amd import lemo

F32, BF16 = 0, 1


@pytest.mark.parametrize("dt", [BF16, F32])
@pytest.mark.parametrize("M", [2048, 4096, 16384, 32768, 50001, 131072, 1 << 20])
@pytest.mark.parametrize("C, V", [(1024, 131072), (1024, 32000), (4096, 131072), (256, 50001)])
def test_the_default_piece(dt, M, C, V):
    size = 2 if dt == BF16 else 4
    need = lemo._bytes("lemo_vocab_loss_grad_workspace_bytes", M, C, V, C, dt, 0)
    columns = min(max(8192, (1 << 28) // (M * size)), (V + 255) // 256 * 256, (1 << 31) // ((M + 1) * size))
    G, plane = (M + 1) * columns * size, 4 * M * C
    turned = 4 * columns * min(C, (M + 63) // 64 * 64) if dt == F32 else 0
    planes = 2 if plane >= 64 << 20 else 32 if dt == BF16 else 64  # dX's sums, of as many parts as the contraction is cut into
    small = 8 * M + 2048
    assert need <= G + turned + planes * plane + small
    # pieces are of one size: the last is not a small rest, and all of them together not much more than the vocabulary
    pieces = -(-V // columns)
    assert need >= (M + 1) * size * (V / pieces - 64) + plane


def test_a_smaller_piece_takes_less():
    for dt, size in ((BF16, 2), (F32, 4)):
        for M in (4096, 131072):
            sizes = [lemo._bytes("lemo_vocab_loss_grad_workspace_bytes", M, 1024, 131072, 1024, dt, piece) for piece in (1024, 2048, 4096)]
            for small, large, columns in zip(sizes, sizes[1:], (1024, 2048)):
                assert large - small >= M * columns * size * 0.9
            assert sizes[0] <= (M + 1) * 1024 * size + 4 * 1024 * 1024 + 4 * M * 1024 * (1 if M > 4096 else 64) + 8 * M + 2048


@pytest.mark.parametrize("dt, most", [(BF16, 12 * 16384 * 1024), (F32, (1 << 29) + 12 * 16384 * 64)])
def test_the_loss(dt, most):
    """Up to 16384 rows at a time: 12 bytes for a row and 128 words; binary32: also a piece of logits."""
    for M in (4096, 16384, 131072, 1 << 22):
        assert lemo._bytes("lemo_vocab_loss_workspace_bytes", M, 1024, 131072, dt) <= most + 4 * 16384 + 2048

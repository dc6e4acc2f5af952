"""Dropout of the widest rows that a 32-bit column count names: columns next to 2^31, whose count must not wrap round."""
import pytest
import torch

from test_dropout import LOW, keep16, philox


@pytest.fixture(scope="module")
def lemo():
    from paper_2501_09767_amd import lemo
    return lemo


def tail(C, n, p, seed, stream):
    """Which of the last n columns of token 0 stay."""
    out = []
    for c in range(C - n, C):
        x = philox((c // 8, 0, stream & LOW, stream >> 32), (seed & LOW, seed >> 32))
        out.append((x[c % 8 // 2] >> (16 * (c % 2)) & 0xffff) < keep16(p))
    return torch.tensor(out)


@pytest.mark.gpu
@pytest.mark.parametrize("C", [2 ** 31 - 8, 2 ** 31 - 2048])
def test_columns_next_to_2_to_the_31(lemo, C):
    n = 3000
    rng = torch.tensor([77, 5], dtype=torch.int64, device="cuda")
    R = torch.ones(1, C, dtype=torch.bfloat16, device="cuda")
    lemo.lemo_dropout_add_grad(R, None, rng, 0.5, 2, R)  # in place: each 0 or 2
    keep = tail(C, n, 0.5, 77, 7)
    assert torch.equal(R[0, C - n:].cpu(), keep.bfloat16() * 2) and torch.equal(R[0, :8].cpu().bool(), tail(8, 8, 0.5, 77, 7))
    kept = sum(int(R[0, i:i + 2 ** 28].bool().sum()) for i in range(0, C, 2 ** 28))
    assert abs(kept - C / 2) < 6 * C ** 0.5  # (twelve deviations)
    sums = torch.ones_like(R)
    lemo.lemo_dropout_add(R, sums, None, rng, 0.5, 2)
    assert torch.equal(sums[0, C - n:].cpu(), keep.bfloat16() * 4 + 1)

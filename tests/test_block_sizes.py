"""Sizes at the ends of what the attention over listed key blocks takes."""
import ctypes

import pytest


@pytest.fixture(scope="module")
def lemo():
    from paper_2501_09767_amd import lemo
    return lemo


def grad_workspace(lemo, S_q, S_k, H, H_kv, d, T, b, bq):
    n = ctypes.c_size_t()
    return lemo._lib.lemo_block_attention_grad_workspace_bytes(S_q, S_k, H, H_kv, d, T, b, bq, ctypes.byref(n)), n.value


def test_gradient_counts_list_entries_in_32_bits(lemo):
    """Places in the lists turned round are 32-bit: 1048544 queries of 32 key heads with 65 blocks each are 2^31 + 33 million.  Refused on the
    host; the addresses are never touched."""
    S, S_k, H, T = 1048544, 2080, 32, 65
    assert S * H * min(T, S_k // 32) >= 2 ** 31
    assert grad_workspace(lemo, S, S_k, H, H, 64, T, 32, 1)[0] == -6
    P = 0x100000
    for S_q, most in ((S, T), (2 ** 31 // (H * 65) + 1, T), (2 ** 31 // (H * 65) + 1, 1000)):  # (a list longer than there are blocks)
        rc = lemo._lib.lemo_block_attention_grad(P, P, P, P, P, P, S_q, S_k, H, H, 64, 1, 0, 64, 0, 64, 0, 64, 0, 64, 0, 64, P, most, 32, 1, 0, 0.0, 1, P, P, P, P,
                                                 1 << 62, None)
        assert rc == -6
    rc, size = grad_workspace(lemo, 2 ** 31 // (H * 65) - 1, S_k, H, H, 64, 65, 32, 1)
    assert rc == 0 and size > 4 * (2 ** 31 - 3 * H * 65)
    # rows of a key block's list: queries times heads of the group
    assert grad_workspace(lemo, 2 ** 25, 32, 64, 1, 64, 1, 32, 64)[0] == -6
    assert grad_workspace(lemo, 2 ** 24, 32, 64, 1, 64, 1, 32, 64)[0] == 0

"""Sizes at the ends of what the attention over listed key blocks takes."""
import ctypes
import math

import pytest
import torch


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


@pytest.mark.gpu
@pytest.mark.parametrize("H,H_kv,d,bq", [(2, 2, 64, 64), (4, 1, 128, 64), (4, 2, 128, 1)])
def test_blocks_of_keys_next_to_2_31(lemo, H, H_kv, d, bq):
    """2^31 - 4097 keys that share one row: the last block, 61439 keys, and the first.  All logits of a query are equal."""
    S_k, b, S_q = 2 ** 31 - 4097, 65536, 70
    g = torch.Generator().manual_seed(d + H)
    Q, k, v = (torch.randn(n, h, d, generator=g).to(torch.bfloat16) for n, h in ((S_q, H), (1, H_kv), (1, H_kv)))
    last = (S_k - 1) // b
    keys = S_k - last * b
    for entry, count in ((last, keys), (0, b), (last + 1, 0)):
        blocks = torch.full((-(-S_q // bq), H_kv, 1), entry, dtype=torch.int32, device="cuda")
        O, lse2 = lemo.lemo_block_attention(Q.cuda(), k.cuda().expand(S_k, H_kv, d), v.cuda().expand(S_k, H_kv, d), blocks, b, bq, 0)
        if count == 0:
            assert not O.any() and (lse2 == -math.inf).all()
            continue
        want = v.double()[0].repeat_interleave(H // H_kv, 0).expand(S_q, H, d)
        # equal values of P, up to 2^8, rounded once: 2^-8; their binary32 sums over `count` keys in chains of count / 16: count / 16 2^-24
        assert ((O.double().cpu() - want).abs() <= (2.0 ** -8 * (2 + 2.0 ** -8) + count * 2.0 ** -27) * want.abs()).all()
        x = (Q.double() * k.double()[0].repeat_interleave(H // H_kv, 0)).sum(2) / math.sqrt(d) * math.log2(math.e) + math.log2(count)
        assert ((lse2.double().cpu().t() - x).abs() <= 2.0 ** -10).all()

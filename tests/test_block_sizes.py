"""Sizes at the ends of what the attention over listed key blocks takes."""
import ctypes
import math

import pytest
import torch

from test_block_attention import chosen64


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


def own_blocks(S_q, S_k, q_start, b, bq):
    """The most blocks that hold positions of one query block's queries, from the definition."""
    return max(len({i // b for i in range(q_start + m, min(q_start + min(m + bq, S_q), S_k))}) for m in range(0, S_q, bq))


# S_q, S_k, q_start, b, bq: query blocks of one, of all queries, shorter and longer than key blocks, across their ends or not, past the keys
OWN = [(100, 100, 0, 128, 100), (40, 40, 0, 64, 64), (300, 300, 0, 128, 300), (100, 200, 100, 128, 1000), (33, 33, 0, 32, 33), (64, 64, 0, 96, 32), (96, 200, 50, 32, 48),
       (90, 90, 0, 32, 40), (50, 20, 0, 32, 50), (64, 40, 500, 32, 16), (20, 70, 60, 32, 7), (1, 1, 0, 32, 1), (500, 500, 0, 96, 36), (65, 200, 32, 32, 64)]


@pytest.mark.gpu
@pytest.mark.parametrize("n", range(len(OWN)))
def test_lists_with_room_for_the_queries_own_blocks_and_no_more(lemo, n):
    S_q, S_k, q_start, b, bq = OWN[n]
    T = max(1, own_blocks(*OWN[n]))
    g = torch.Generator().manual_seed(n)
    Q, means = torch.randn(S_q, 4, 64, generator=g).to(torch.bfloat16), torch.randn(-(-S_k // b), 2, 64, generator=g)
    for room in (T, T + 1):
        got = lemo.lemo_select_blocks(Q.cuda(), means.cuda(), S_k, b, bq, room, q_start=q_start)
        assert torch.equal(got.cpu(), chosen64(Q, means, S_k, b, bq, room, True, q_start))
    if T > 1:
        with pytest.raises(lemo.LemoError):
            lemo.lemo_select_blocks(Q.cuda(), means.cuda(), S_k, b, bq, T - 1, q_start=q_start)


def test_refused_where_the_own_blocks_do_not_fit():
    """On the host alone: addresses are never touched."""
    from paper_2501_09767_amd import lemo
    for S_q, S_k, q_start, b, bq in OWN:
        for T in range(1, own_blocks(S_q, S_k, q_start, b, bq)):
            rc = lemo._lib.lemo_select_blocks(0x100000, S_q, 4, 2, 64, 1, 256, 64, 0x200000, S_k, q_start, b, bq, T, 1, 0x300000, None)
            assert rc == -2, (S_q, S_k, q_start, b, bq, T)
    # (blocks of 65536 keys, 12345 queries each: only the sixth block of them goes across an end)
    f = lambda S, T: lemo._lib.lemo_select_blocks(0x100000, S, 4, 2, 64, 1, 256, 64, 0x200000, S, 0, 65536, 12345, T, 1, 0x300000, None)  # noqa: E731
    assert f(12345 * 6, 1) == -2

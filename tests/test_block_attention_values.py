"""Attention over listed key blocks: values at the ends of what a type holds, scales of the caller's.  Bounds as in test_block_attention.py."""
import math

import pytest
import torch

import test_block_attention as base
from test_block_attention import HALF, close, draw, lists

BAD = [math.nan, math.inf, -math.inf]


@pytest.fixture(scope="module")
def lemo():
    from paper_2501_09767_amd import lemo
    return lemo


@pytest.mark.gpu
@pytest.mark.parametrize("where", ["K", "V"])
@pytest.mark.parametrize("S,H,H_kv,d,b,bq,causal", [(200, 4, 4, 64, 32, 1, True), (200, 8, 2, 128, 32, 1, True), (150, 2, 2, 128, 64, 3, False), (333, 16, 4, 64, 32, 2, False),
                                                    (600, 16, 16, 128, 32, 1, True)])
def test_blocks_that_only_other_queries_list(lemo, S, H, H_kv, d, b, bq, causal, where):
    """Lists of few rows are worked on together.  One key block holds what is not finite; every third list names it, the other queries'
    results are those of a run in which it holds zeros."""
    case = base._c(S, S, H, H_kv, d, b, bq, 3, causal=causal)
    Q, K, V, dO = draw(S + d, (S, H, d), (S, H_kv, d), (S, H_kv, d), (S, H, d))
    n_qb, bad = -(-S // bq), 1
    blocks = torch.full((n_qb, H_kv, 3), -1, dtype=torch.int32)
    for m in range(n_qb):
        last = min((min((m + 1) * bq, S) - 1) // b, (S - 1) // b) if causal else (S - 1) // b
        others = [n for n in range(last + 1) if n != bad]
        for g in range(H_kv):
            pick = sorted({others[(m + g) % len(others)], others[-1]} | ({bad} if (m + g) % 3 == 0 and last >= bad else set()))
            blocks[m, g, :len(pick)] = torch.tensor(pick, dtype=torch.int32)
    spoiled = (blocks == bad).any(2).repeat_interleave(bq, 0)[:S].repeat_interleave(H // H_kv, 1)  # [S,H]
    assert spoiled.any() and not spoiled.all()
    for x in (K, V):
        x[bad * b:(bad + 1) * b] = 0
    K2, V2 = K.clone(), V.clone()
    target = K2 if where == "K" else V2
    for i, value in enumerate(BAD):
        target[bad * b + 5 * i:bad * b + 5 * i + 3, :, i::7] = value
    flags = lemo.CAUSAL if causal else 0
    q, do, bl = Q.cuda(), dO.cuda(), blocks.cuda()
    O, lse2 = lemo.lemo_block_attention(q, K.cuda(), V.cuda(), bl, b, bq, flags)
    O2, lse2_2 = lemo.lemo_block_attention(q, K2.cuda(), V2.cuda(), bl, b, bq, flags)
    ref = base.reference(case, Q, K, V, blocks, dO, O.cpu())
    clear = ~spoiled
    off = (O2.double().cpu() - ref["O"]).abs() - (HALF * ref["O"].abs() + (1 + HALF) * (HALF + 4 * ref["E"] + 2.0 ** -14)[..., None] * ref["O_mag"])
    assert off[clear].max() <= 1e-30  # (a NaN is no smaller)
    assert torch.equal(O2.cpu()[clear], O.cpu()[clear]) and torch.equal(lse2_2.cpu().t()[clear], lse2.cpu().t()[clear])
    if where == "V":
        assert not torch.isfinite(O2.cpu()[spoiled & (torch.arange(S) >= (bad + 1) * b)[:, None]]).all()
    grads = lemo.lemo_block_attention_grad(do, q, K2.cuda(), V2.cuda(), O2, lse2_2, bl, b, bq, flags)
    off = (grads[0].double().cpu() - ref["dQ"]).abs() - (HALF * ref["dQ"].abs() + (1 + HALF) * ref["dQ_mag"] * (1 + 2.0 ** -10))
    assert off[clear].max() <= 1e-30
    # key blocks that no spoiled query lists
    for g in range(H_kv):
        for n in range(-(-S // b)):
            naming = (blocks[:, g] == n).any(1)
            if n == bad or ((blocks[:, g] == bad).any(1) & naming).any():
                continue
            at = slice(n * b, (n + 1) * b)
            for name, got in (("dK", grads[1]), ("dV", grads[2])):
                off = (got.double().cpu()[at, g] - ref[name][at, g]).abs() - (HALF * ref[name][at, g].abs() + (1 + HALF) * ref[name + "_mag"][at, g] * (1 + 2.0 ** -10))
                assert off.max() <= 1e-30, (name, g, n)


@pytest.mark.gpu
@pytest.mark.parametrize("H,H_kv,d,S,bq", [(4, 1, 128, 640, 64), (80, 20, 128, 640, 64), (2, 2, 128, 640, 64), (4, 1, 64, 640, 64), (8, 2, 128, 320, 1)])
def test_later_logits_within_the_range_of_the_reference_and_large_values(lemo, H, H_kv, d, S, bq):
    """Later logits up to 2^97 above the first ones, values of 2^40: their products pass the range of binary32, their quotient does not."""
    case = base._c(S, S, H, H_kv, d, 32, bq, 16)
    Q, K, V = draw(5, (S, H, d), (S, H_kv, d), (S, H_kv, d))
    V = V * 2.0 ** 40
    blocks = torch.full((-(-S // bq), H_kv, 16), -1, dtype=torch.int32)
    for m in range(len(blocks)):
        last = (min((m + 1) * bq, S) - 1) // 32
        pick = list(range(last + 1))[-16:]
        blocks[m, :, :len(pick)] = torch.tensor(pick, dtype=torch.int32)
    Q[::3] = 4.0
    K *= 0.125
    K[149::150] = 94.0 / (4.0 * d / math.sqrt(d) * math.log2(math.e))  # one key in 150: 94 (and its rounding to bf16) for these queries
    O, lse2 = lemo.lemo_block_attention(Q.cuda(), K.cuda(), V.cuda(), blocks.cuda(), 32, bq)
    ref = base.reference(case, Q, K, V, blocks)
    assert 90 < ref["lse2"].max() < 100
    base.check_forward(O, lse2, ref)


@pytest.mark.gpu
@pytest.mark.parametrize("n", range(7))
def test_scales_of_the_caller(lemo, n):
    case, scale = [
        (base._c(257, 257, 8, 2, 128, 64, 64, 4), 0.2),                              # 256 rows a list
        (base._c(300, 300, 4, 2, 128, 32, 48, 4), 0.03),                             # 96
        (base._c(161, 161, 4, 2, 64, 32, 16, 4, causal=False), 0.25),                # 32
        (base._c(130, 300, 8, 1, 128, 32, 1, 5, q_start=170), 0.11),                 # lists together
        (base._c(200, 200, 4, 4, 64, 64, 1, 3), 0.3),
        (base._c(1, 3000, 8, 2, 128, 64, 1, 16, q_start=2999), 0.17),                # one list, several workgroups
        (base._c(64, 4000, 4, 2, 128, 64, 64, 30, q_start=3936), 0.05),
    ][n]
    print(case, scale, flush=True)
    S_q, S_k, H, H_kv, d, b, bq = (case[k] for k in ("S_q", "S_k", "H", "H_kv", "d", "b", "bq"))
    Q, K, V, dO = draw(n + 40, (S_q, H, d), (S_k, H_kv, d), (S_k, H_kv, d), (S_q, H, d))
    blocks = lists(case, "own", n)
    flags = lemo.CAUSAL if case["causal"] else 0
    x = [t.cuda() for t in (Q, K, V, blocks, dO)]
    O, lse2 = lemo.lemo_block_attention(*x[:4], b, bq, flags, scale, case["q_start"])
    # the definition takes 1 / sqrt(d): the same logits from queries that are larger by scale sqrt(d), in 64 bits
    factor = scale * math.sqrt(d)
    ref = base.reference(case, Q.double() * factor, K, V, blocks, dO, O.cpu())
    ref["dQ"], ref["dQ_mag"] = ref["dQ"] * factor, ref["dQ_mag"] * factor
    base.check_forward(O, lse2, ref)
    base.check_grads(lemo.lemo_block_attention_grad(x[4], *x[:3], O, lse2, x[3], b, bq, flags, scale, case["q_start"]), ref)


@pytest.mark.gpu
@pytest.mark.parametrize("H,H_kv,d,b,T,S,lengths,scale", [(8, 2, 128, 64, 4, 500, [500, 1, 64, 449, 0], 0.2), (4, 4, 64, 32, 3, 200, [97, 200], 0.02)])
def test_scales_of_the_caller_single_tokens(lemo, H, H_kv, d, b, T, S, lengths, scale):
    B = len(lengths)
    Q, K, V = draw(H + T, (B, H, d), (B, S, H_kv, d), (B, S, H_kv, d))
    blocks = torch.full((B, H_kv, T), -1, dtype=torch.int32)
    for s, n in enumerate(lengths):
        pick = list(range(-(-n // b)))[-T:]
        blocks[s, :, :len(pick)] = torch.tensor(pick, dtype=torch.int32)
    O = lemo.lemo_block_attention_step(Q.cuda(), K.cuda(), V.cuda(), torch.tensor(lengths, dtype=torch.int32, device="cuda"), blocks.cuda(), b, scale)
    for s, n in enumerate(lengths):
        if n == 0:
            assert not O[s].any()
            continue
        case = base._c(1, n, H, H_kv, d, b, 1, T, q_start=n - 1)
        ref = base.reference(case, Q[s:s + 1].double() * (scale * math.sqrt(d)), K[s, :n], V[s, :n], blocks[s:s + 1])
        close("O", O[s:s + 1], ref["O"], HALF * ref["O"].abs() + (1 + HALF) * (HALF + 4 * ref["E"] + 2.0 ** -14)[..., None] * ref["O_mag"])


@pytest.mark.gpu
@pytest.mark.parametrize("n", range(8))
def test_what_lies_behind_the_last_query(lemo, n):
    """A part of a prompt over a cache that has room for more: what stands there is nobody's key yet, NaN among it."""
    case = [
        base._c(70, 300, 8, 2, 128, 64, 64, 4, q_start=100),      # 256 rows a list
        base._c(300, 500, 80, 20, 128, 32, 48, 6, q_start=23),    # and more tiles than there are workgroups
        base._c(90, 200, 4, 2, 128, 32, 48, 4, q_start=37),       # 96 rows
        base._c(45, 128, 4, 2, 64, 32, 16, 3, q_start=40),        # 32
        base._c(77, 140, 8, 1, 128, 32, 1, 4, q_start=20),        # lists together
        base._c(50, 90, 4, 4, 64, 64, 1, 2, q_start=0),
        base._c(1, 3000, 8, 2, 128, 64, 1, 16, q_start=1999),     # one list, several workgroups
        base._c(130, 333, 6, 2, 128, 128, 5, 2, q_start=66),
    ][n]
    print(case, flush=True)
    S_q, S_k, H, H_kv, d, b, bq = (case[k] for k in ("S_q", "S_k", "H", "H_kv", "d", "b", "bq"))
    Q, K, V, dO = draw(n + 60, (S_q, H, d), (S_k, H_kv, d), (S_k, H_kv, d), (S_q, H, d))
    blocks = lists(case, "own", n)
    blocks[0, :, -1] = (S_k - 1) // b  # (a list that names blocks behind its queries as well)
    end = case["q_start"] + S_q
    K2, V2 = K.clone(), V.clone()
    for x in (K2, V2):
        x[end:] = torch.tensor(BAD)[torch.arange(S_k - end) % 3][:, None, None].to(torch.bfloat16)
    x = [t.cuda() for t in (Q, K2, V2, blocks, dO)]
    O, lse2 = lemo.lemo_block_attention(*x[:4], b, bq, q_start=case["q_start"])
    ref = base.reference(case, Q, K, V, blocks, dO, O.cpu())
    base.check_forward(O, lse2, ref)
    grads = lemo.lemo_block_attention_grad(x[4], *x[:3], O, lse2, x[3], b, bq, q_start=case["q_start"])
    base.check_grads(grads, ref)
    assert not grads[1][end:].any() and not grads[2][end:].any()

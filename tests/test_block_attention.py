"""Attention over key blocks that a list names for every query block: the choice, the attention, its gradients and the form for single
tokens, against the definitions in 64 bits.

Tolerances.  A bf16 value is off by at most half a step, 2^-8 of it.  With E = (d + 8) 2^-24 max_j sum_c |q_c k_jc| scale log2(e) for the
binary32 logits, a probability is off by at most 4 E + 2^-14 of it (logit, exponential, normaliser) and, where it goes into a product, by
2^-8 for its rounding to bf16; so O by 2^-8 |o| + (2^-8 + 4 E + 2^-14) sum_j P_j |V_j| (1 + 2^-8), and the gradients likewise with the
magnitudes of their own terms.  dP and delta are binary32 sums of d products: (d + 8) 2^-24 of their terms' magnitudes."""
import ctypes
import math

import pytest
import torch

HALF = 2.0 ** -8


@pytest.fixture(scope="module")
def lemo():
    from paper_2501_09767_amd import lemo
    return lemo


def draw(seed, *shapes, std=1.0):
    g = torch.Generator().manual_seed(seed)
    return [(torch.randn(*s, generator=g) * std).to(torch.bfloat16) for s in shapes]


def allowed(case, blocks):
    """[query blocks -> dense mask]: [S_q, H_kv, S_k] from the rule for lists."""
    S_q, S_k, b, bq = case["S_q"], case["S_k"], case["b"], case["bq"]
    nb = -(-S_k // b)
    mask = torch.zeros(S_q, blocks.shape[1], S_k, dtype=torch.bool)
    for m, per_head in enumerate(blocks.tolist()):
        for g, entries in enumerate(per_head):
            top = -1
            for n in entries:
                if 0 <= n < nb and n > top:
                    top = n
                    mask[m * bq:(m + 1) * bq, g, n * b:(n + 1) * b] = True
    if case["causal"]:
        mask &= (torch.arange(S_k) <= case["q_start"] + torch.arange(S_q)[:, None])[:, None]
    return mask


def reference(case, Q, K, V, blocks, dO=None, O=None):
    H, H_kv, d = case["H"], case["H_kv"], case["d"]
    scale = 1 / math.sqrt(d)
    mask = allowed(case, blocks)
    q, k, v = (x.double() for x in (Q, K, V))
    out = dict(O=torch.zeros_like(q), O_mag=torch.zeros_like(q), lse2=torch.full((H, len(q)), -math.inf, dtype=torch.float64), E=torch.zeros(len(q), H, dtype=torch.float64))
    if dO is not None:
        do = dO.double()
        for n, like in (("dQ", q), ("dK", k), ("dV", v)):
            out[n], out[n + "_mag"] = torch.zeros_like(like), torch.zeros_like(like)
    for h in range(H):
        g = h * H_kv // H
        x = (q[:, h] @ k[:, g].T * scale).masked_fill(~mask[:, g], -math.inf)
        E = (d + 8) * 2.0 ** -24 * scale * 1.4427 * (q[:, h].abs() @ k[:, g].abs().T).masked_fill(~mask[:, g], 0).amax(1)
        P = torch.softmax(x, 1).nan_to_num(0.0)
        out["lse2"][h] = torch.logsumexp(x, 1) / math.log(2)
        out["O"][:, h], out["O_mag"][:, h], out["E"][:, h] = P @ v[:, g], P @ v[:, g].abs(), E
        if dO is None:
            continue
        dP, size = do[:, h] @ v[:, g].T, do[:, h].abs() @ v[:, g].abs().T
        delta, dsize = (do[:, h] * O[:, h].double()).sum(1, keepdim=True), (do[:, h] * O[:, h].double()).abs().sum(1, keepdim=True)
        dS = P * (dP - delta)
        off = (HALF + 4 * E + 2.0 ** -14)[:, None]
        err = dS.abs() * off + P * (size + dsize) * (d + 8) * 2.0 ** -24 * (1 + off)
        out["dQ"][:, h], out["dQ_mag"][:, h] = scale * dS @ k[:, g], scale * err @ k[:, g].abs()
        out["dK"][:, g] += scale * dS.T @ q[:, h]
        out["dK_mag"][:, g] += scale * err.T @ q[:, h].abs()
        out["dV"][:, g] += P.T @ do[:, h]
        out["dV_mag"][:, g] += (P * off).T @ do[:, h].abs()
    return out


def close(name, got, want, bound):
    got = got.double().cpu()
    assert got.shape == want.shape and torch.isfinite(got).all(), name
    off = (got - want).abs() - bound
    assert off.max() <= 1e-30, f"{name}: {off.max().item():.3g} over the bound at {int(off.argmax())}"


def check_forward(got_O, got_lse, ref):
    E = ref["E"]
    close("O", got_O, ref["O"], HALF * ref["O"].abs() + (1 + HALF) * (HALF + 4 * E + 2.0 ** -14)[..., None] * ref["O_mag"])
    lse, want = got_lse.double().cpu(), ref["lse2"]
    assert torch.equal(torch.isinf(lse), torch.isinf(want))
    there = ~torch.isinf(want)
    assert ((lse - want).abs()[there] <= (2 * E.T + 2.0 ** -20 + 2.0 ** -22 * want.abs())[there]).all()


def check_grads(grads, ref):
    for name, got in zip(("dQ", "dK", "dV"), grads):
        close(name, got, ref[name], HALF * ref[name].abs() + (1 + HALF) * ref[name + "_mag"] * (1 + 2.0 ** -10))


def lists(case, kind, seed):
    """kind: 'own' the queries' own blocks and others, ascending; 'any' entries of every sort; 'first' block 0 on every list; 'none'."""
    g = torch.Generator().manual_seed(seed)
    n_qb, nb, T = -(-case["S_q"] // case["bq"]), -(-case["S_k"] // case["b"]), case["T"]
    if kind == "none":
        return torch.full((n_qb, case["H_kv"], T), -1, dtype=torch.int32)
    if kind == "any":
        return torch.randint(-2, nb + 2, (n_qb, case["H_kv"], T), generator=g, dtype=torch.int32)
    out = torch.full((n_qb, case["H_kv"], T), -1, dtype=torch.int32)
    for m in range(n_qb):
        last = (case["q_start"] + min((m + 1) * case["bq"], case["S_q"]) - 1) // case["b"]
        last = min(last, nb - 1) if case["causal"] else nb - 1
        for k in range(case["H_kv"]):
            pick = torch.randperm(last + 1, generator=g)[:T].tolist()
            if kind == "first":
                pick = [0] + [n for n in pick if n][:T - 1]
            elif last not in pick:
                pick[-1] = last
            out[m, k, :len(pick)] = torch.tensor(sorted(pick), dtype=torch.int32)
    return out


def _c(S_q, S_k, H, H_kv, d, b, bq, T, q_start=0, causal=True, kind="own"):
    return dict(S_q=S_q, S_k=S_k, H=H, H_kv=H_kv, d=d, b=b, bq=bq, T=T, q_start=q_start, causal=causal, kind=kind)


CASES = [
    _c(1, 1, 1, 1, 64, 32, 1, 1),
    _c(1, 1, 2, 1, 128, 64, 64, 3),
    _c(100, 100, 4, 4, 64, 32, 16, 3),
    _c(257, 257, 8, 2, 128, 64, 64, 4),
    _c(130, 513, 8, 1, 128, 32, 1, 5, q_start=383),
    _c(70, 300, 6, 3, 64, 96, 32, 2, causal=False),
    _c(90, 333, 4, 2, 128, 32, 1, 7, causal=False, kind="any"),
    _c(161, 161, 4, 2, 64, 64, 3, 70, kind="any"),
    _c(300, 300, 4, 2, 128, 128, 300, 3),
    _c(300, 300, 4, 1, 128, 128, 1000, 2),
    _c(65, 200, 40, 1, 64, 32, 8, 6, q_start=135),
    _c(200, 200, 16, 8, 64, 64, 16, 4),
    _c(96, 200, 16, 16, 128, 32, 48, 6, q_start=50),
    _c(700, 700, 2, 1, 64, 32, 1, 4, kind="first"),
    _c(600, 600, 2, 2, 128, 64, 1, 3, kind="first"),
    _c(40, 64, 4, 2, 128, 32, 8, 2, q_start=24, kind="none"),
    _c(64, 40, 4, 2, 64, 32, 16, 2, q_start=500),
    # more tiles of 256 rows than there are CUs: a workgroup walks over several lists
    _c(700, 700, 80, 20, 128, 32, 48, 9),
    _c(330, 500, 72, 24, 128, 64, 50, 6, q_start=100, kind="any"),
    _c(250, 300, 96, 48, 128, 32, 100, 12, causal=False, kind="any"),
    _c(400, 400, 66, 33, 128, 32, 70, 5, kind="none"),
    # rows of a key block's list that do not divide what a workgroup takes at a time; more query blocks than a wave takes words of
    _c(333, 333, 6, 2, 128, 128, 5, 3),
    _c(333, 400, 5, 1, 64, 128, 7, 2, q_start=67),
    _c(150, 290, 14, 2, 128, 96, 11, 2, causal=False, kind="any"),
    _c(2150, 2150, 2, 1, 64, 32, 1, 3),
]


@pytest.mark.gpu
@pytest.mark.parametrize("n", range(len(CASES)))
def test_attention_and_gradients_against_64_bits(lemo, n):
    case = CASES[n]
    print(case, flush=True)
    Q, K, V, dO = draw(n, (case["S_q"], case["H"], case["d"]), (case["S_k"], case["H_kv"], case["d"]), (case["S_k"], case["H_kv"], case["d"]),
                       (case["S_q"], case["H"], case["d"]))
    K[::7] *= 3  # a few keys that many queries look for
    blocks = lists(case, case["kind"], n)
    flags = lemo.CAUSAL if case["causal"] else 0
    d = [x.cuda() for x in (Q, K, V, blocks, dO)]
    O, lse2 = lemo.lemo_block_attention(d[0], d[1], d[2], d[3], case["b"], case["bq"], flags, q_start=case["q_start"])
    ref = reference(case, Q, K, V, blocks, dO, O.cpu())
    check_forward(O, lse2, ref)
    grads = lemo.lemo_block_attention_grad(d[4], d[0], d[1], d[2], O, lse2, d[3], case["b"], case["bq"], flags, q_start=case["q_start"])
    check_grads(grads, ref)
    again = lemo.lemo_block_attention_grad(d[4], d[0], d[1], d[2], O, lse2, d[3], case["b"], case["bq"], flags, q_start=case["q_start"])
    assert all(torch.equal(x, y) for x, y in zip(grads, again))


@pytest.mark.gpu
@pytest.mark.parametrize("H,H_kv,d,S,bq", [(4, 1, 128, 640, 64), (80, 20, 128, 640, 64), (2, 2, 128, 640, 64), (4, 1, 64, 640, 64), (8, 2, 128, 320, 1)])
def test_keys_that_outgrow_the_first_ones(lemo, H, H_kv, d, S, bq):
    """Logits whose later values lie hundreds above the first: references that a first stage left have to give way."""
    case = _c(S, S, H, H_kv, d, 32, bq, 16)
    Q, K, V = draw(3, (S, H, d), (S, H_kv, d), (S, H_kv, d))
    blocks = torch.full((-(-S // bq), H_kv, 16), -1, dtype=torch.int32)
    for m in range(len(blocks)):
        last = (min((m + 1) * bq, S) - 1) // 32
        pick = list(range(last + 1))[-16:]
        blocks[m, :, :len(pick)] = torch.tensor(pick, dtype=torch.int32)
    # every third query looks along one direction, and one key in 150 lies far out along it
    Q[::3] = 4.0
    K[149::150] = 30.0 * torch.linspace(0.2, 1.0, len(K[149::150]))[:, None, None].to(torch.bfloat16)
    O, lse2 = lemo.lemo_block_attention(Q.cuda(), K.cuda(), V.cuda(), blocks.cuda(), 32, bq)
    ref = reference(case, Q, K, V, blocks)
    assert ref["lse2"].max() - ref["lse2"].min() > 150
    check_forward(O, lse2, ref)


@pytest.mark.gpu
def test_gradients_against_differences(lemo):
    """Differences of the definition in 64 bits, along random directions.  The gradients are off by what check_grads bounds; along a
    direction of unit entries that is at most the sum of the bounds, and half a per cent of the terms' size is far above it."""
    case = _c(48, 48, 4, 2, 64, 32, 16, 2)
    Q, K, V, dO = draw(31, (48, 4, 64), (48, 2, 64), (48, 2, 64), (48, 4, 64))
    blocks = lists(case, "own", 31)
    mask = allowed(case, blocks)

    def loss(q, k, v):
        total = 0.0
        for h in range(4):
            x = (q[:, h] @ k[:, h // 2].T / 8).masked_fill(~mask[:, h // 2], -math.inf)
            total = total + ((torch.softmax(x, 1) @ v[:, h // 2]) * dO[:, h].double()).sum()
        return total.item()

    d = [x.cuda() for x in (Q, K, V, blocks, dO)]
    O, lse2 = lemo.lemo_block_attention(d[0], d[1], d[2], d[3], 32, 16)
    grads = [g.double().cpu() for g in lemo.lemo_block_attention_grad(d[4], d[0], d[1], d[2], O, lse2, d[3], 32, 16)]
    at = [Q.double(), K.double(), V.double()]
    g = torch.Generator().manual_seed(1)
    for i in range(3):
        for _ in range(3):
            e = torch.randn(at[i].shape, generator=g, dtype=torch.float64)
            step = [1e-5 * e if j == i else 0.0 for j in range(3)]
            slope = (loss(*(x + s for x, s in zip(at, step))) - loss(*(x - s for x, s in zip(at, step)))) / 2e-5
            terms = grads[i] * e
            assert abs(slope - terms.sum().item()) <= 0.005 * terms.abs().sum().item()


@pytest.mark.gpu
def test_operands_inside_larger_tensors(lemo):
    """Q, K, V as slices of one projection's result; results into slices too."""
    case = _c(150, 150, 8, 2, 64, 32, 16, 3)
    qkv, = draw(2, (150, 12, 64))
    blocks, big = lists(case, "own", 2).cuda(), qkv.cuda()
    q, k, v = big[:, :8], big[:, 8:10], big[:, 10:]
    O, lse2 = lemo.lemo_block_attention(q, k, v, blocks, 32, 16)
    O1, lse1 = lemo.lemo_block_attention(q.contiguous(), k.contiguous(), v.contiguous(), blocks, 32, 16)
    wide = torch.full((150, 16, 64), 5.0, dtype=torch.bfloat16, device="cuda")
    O2, _ = lemo.lemo_block_attention(q, k, v, blocks, 32, 16, O=wide[:, 4:12])
    assert torch.equal(O, O1) and torch.equal(lse2, lse1) and torch.equal(O, O2) and (wide[:, :4] == 5).all() and (wide[:, 12:] == 5).all()
    dO = torch.randn(8, 150, 64, device="cuda").to(torch.bfloat16).transpose(0, 1)  # heads first in memory
    got = lemo.lemo_block_attention_grad(dO, q, k, v, wide[:, 4:12], lse2, blocks, 32, 16)
    want = lemo.lemo_block_attention_grad(dO.contiguous(), q.contiguous(), k.contiguous(), v.contiguous(), O, lse2, blocks, 32, 16)
    assert all(torch.equal(x, y) for x, y in zip(got, want))


def chosen64(Q, means, S_k, b, bq, T, causal, q_start):
    S, H, d = Q.shape
    nb, H_kv = means.shape[:2]
    out = torch.full((-(-S // bq), H_kv, T), -1, dtype=torch.int32)
    for m in range(len(out)):
        rows = Q[m * bq:(m + 1) * bq].double()
        first, last = q_start + m * bq, min(q_start + m * bq + len(rows) - 1, S_k - 1)
        for g in range(H_kv):
            s = (means[:, g].double() @ rows[:, g * H // H_kv:(g + 1) * H // H_kv].sum((0, 1))).tolist()
            order = list(range(nb))
            if causal:
                order = [n for n in order if n * b <= last]
                s = [math.inf if n * b + b > first else x for n, x in enumerate(s)]
            pick = sorted(sorted(order, key=lambda n: (-s[n], n))[:T])
            out[m, g, :len(pick)] = torch.tensor(pick, dtype=torch.int32)
    return out


@pytest.mark.gpu
@pytest.mark.parametrize("S_q,S_k,H,H_kv,d,b,bq,T,causal,q_start,dtype", [
    (1, 1, 1, 1, 64, 32, 1, 1, True, 0, torch.bfloat16),
    (1, 5000, 8, 2, 128, 64, 1, 16, True, 4999, torch.bfloat16),
    (333, 333, 8, 8, 64, 32, 16, 5, True, 0, torch.bfloat16),
    (500, 500, 6, 3, 128, 64, 64, 20, True, 0, torch.float32),
    (100, 3000, 4, 1, 64, 32, 24, 9, True, 2900, torch.bfloat16),
    (100, 1000, 4, 2, 128, 96, 7, 3, False, 0, torch.float32),
    (64, 30, 2, 1, 64, 32, 16, 4, True, 200, torch.bfloat16),
    (40, 9000, 2, 2, 64, 32, 8, 100, False, 17, torch.bfloat16),
    (600, 600, 16, 16, 64, 32, 1, 5, True, 0, torch.bfloat16),       # thousands of lists of few rows: several to a workgroup
    (530, 6000, 32, 16, 128, 32, 1, 12, True, 5400, torch.bfloat16),
    (300, 5000, 8, 8, 64, 32, 1, 9, False, 0, torch.float32),
])
def test_means_and_choice_against_64_bits(lemo, S_q, S_k, H, H_kv, d, b, bq, T, causal, q_start, dtype):
    g = torch.Generator().manual_seed(S_q + S_k)
    Q, K = torch.randn(S_q, H, d, generator=g).to(dtype), torch.randn(S_k, H_kv, d, generator=g).to(dtype)
    means = lemo.lemo_block_means(K.cuda(), b)
    want = torch.stack([x.double().mean(0) for x in K.split(b)])
    assert ((means.double().cpu() - want).abs() <= 2.0 ** -24 * want.abs() * (1 + 1e-6)).all()
    blocks = lemo.lemo_select_blocks(Q.cuda(), means, S_k, b, bq, T, lemo.CAUSAL if causal else 0, q_start)
    assert torch.equal(blocks.cpu(), chosen64(Q, means.cpu(), S_k, b, bq, T, causal, q_start))


@pytest.mark.gpu
def test_choice_of_ties_and_of_what_is_not_a_number(lemo):
    Q = torch.ones(10, 2, 64, dtype=torch.bfloat16, device="cuda")
    means = torch.zeros(200, 1, 64, device="cuda")
    means[::2] *= -1.0  # -0 ties +0
    got = lemo.lemo_select_blocks(Q, means, 200 * 32, 32, 10, 5, 0)
    assert got.tolist() == [[[0, 1, 2, 3, 4]]]
    means[[7, 150]] = 1.0
    got = lemo.lemo_select_blocks(Q, means, 200 * 32, 32, 10, 5, 0)
    assert got.tolist() == [[[0, 1, 2, 7, 150]]]
    # many lists, all scores equal, and equal but in the last bits of their upper halves
    Q = torch.ones(600, 16, 64, dtype=torch.bfloat16, device="cuda")
    same = torch.ones(40, 16, 64, device="cuda")
    assert (lemo.lemo_select_blocks(Q, same, 40 * 32, 32, 1, 6, 0) == torch.arange(6, device="cuda")).all()
    same += torch.arange(40, device="cuda")[:, None, None] * 2.0 ** -23
    assert (lemo.lemo_select_blocks(Q, same, 40 * 32, 32, 1, 6, 0) == torch.arange(34, 40, device="cuda")).all()
    Q = torch.ones(10, 2, 64, dtype=torch.bfloat16, device="cuda")
    for bad in (math.nan, math.inf, -math.inf):
        means[3:100] = bad
        means[50, 0, 5] = -bad
        got = lemo.lemo_select_blocks(Q, means, 200 * 32, 32, 10, 64, lemo.CAUSAL, 6000).cpu()
        assert ((got >= 0) & (got < 200)).all() and (got[..., 1:] > got[..., :-1]).all() and 187 in got.tolist()[0][0]


@pytest.mark.gpu
@pytest.mark.parametrize("H,H_kv,d,b,T,S,lengths", [
    (8, 2, 128, 64, 4, 500, [500, 1, 64, 65, 0, 449, 128, -3, 900]),
    (4, 4, 64, 32, 3, 200, [97, 96]),
    (32, 8, 128, 64, 16, 3000, [3000]),
    (16, 1, 64, 96, 5, 1000, [1000, 31, 480] * 20),
    (160, 1, 128, 32, 4, 300, [300, 77, 64, 0]),
])
def test_single_tokens(lemo, H, H_kv, d, b, T, S, lengths):
    B, nb = len(lengths), -(-S // b)
    Q, K, V = draw(H + S, (B, H, d), (B, S, H_kv, d), (B, S, H_kv, d))
    true = [min(max(n, 0), S) for n in lengths]
    for s, n in enumerate(true):  # what lies behind a sequence is not used
        K[s, n:], V[s, n:] = math.nan, math.nan
    dev = torch.tensor(lengths, dtype=torch.int32, device="cuda")
    Kd, Vd, Qd = K.cuda(), V.cuda(), Q.cuda()
    means = torch.full((B, nb, H_kv, d), math.nan, device="cuda")
    for s, n in enumerate(true):  # blocks that were filled before, as the loop of tokens leaves them
        for k in range(1, n // b + 1):
            at = torch.zeros(B, dtype=torch.int32, device="cuda")
            at[s] = k * b
            lemo.lemo_block_means_step(Kd, at, b, means)
    untouched = means.clone()
    lemo.lemo_block_means_step(Kd, dev, b, means)
    assert torch.equal(torch.nan_to_num(untouched), torch.nan_to_num(means))
    for s, n in enumerate(true):
        if n >= b:
            assert torch.equal(means[s, :n // b], lemo.lemo_block_means(Kd[s, :n // b * b], b))
        assert torch.isnan(means[s, n // b:]).all()
    blocks = lemo.lemo_select_blocks_step(Qd, means, dev, b, T, S_max=S)
    O = lemo.lemo_block_attention_step(Qd, Kd, Vd, dev, blocks, b)
    for s, n in enumerate(true):
        if n == 0:
            assert (blocks[s] == -1).all() and not O[s].any()
            continue
        case = _c(1, n, H, H_kv, d, b, 1, T, q_start=n - 1)
        mine = means[s, :-(-n // b)].cpu().nan_to_num(0.0)
        assert torch.equal(blocks[s].cpu(), chosen64(Q[s:s + 1], mine, n, b, 1, T, True, n - 1)[0])
        ref = reference(case, Q[s:s + 1], K[s, :n], V[s, :n], blocks[s:s + 1].cpu())
        close("O", O[s:s + 1], ref["O"], HALF * ref["O"].abs() + (1 + HALF) * (HALF + 4 * ref["E"] + 2.0 ** -14)[..., None] * ref["O_mag"])


@pytest.mark.gpu
@pytest.mark.parametrize("B", [300, 1100])
def test_choice_for_many_sequences(lemo, B):
    """As for eight of them at a time."""
    H, d, b, T, S = 8, 64, 32, 3, 200
    Q = draw(B, (B, H, d))[0].cuda()
    means = draw(B + 1, (B, 7, H, d))[0].float().cuda()
    lengths = (torch.arange(B, dtype=torch.int32, device="cuda") * 37) % (S + 1)
    got = lemo.lemo_select_blocks_step(Q, means, lengths, b, T, S_max=S)
    for s in range(0, B, 8):
        assert torch.equal(got[s:s + 8], lemo.lemo_select_blocks_step(Q[s:s + 8], means[s:s + 8], lengths[s:s + 8], b, T, S_max=S)), s


@pytest.mark.gpu
def test_caches_beyond_32_bit_offsets(lemo):
    """One sequence of 2.3 million tokens, 8 x 128: its far end lies 4.7 GB behind its begin."""
    S, H, H_kv, d, b = 2_300_000, 8, 8, 128, 64
    K = torch.zeros(1, S, H_kv, d, dtype=torch.bfloat16, device="cuda")
    V = torch.zeros(1, S, H_kv, d, dtype=torch.bfloat16, device="cuda")
    listed = [3, 17000, 33000, (S - 1) // b]
    Q, k, v = draw(8, (1, H, d), (4, b, H_kv, d), (4, b, H_kv, d))
    tok = torch.cat([torch.arange(n * b, min((n + 1) * b, S)) for n in listed])
    k, v = k.view(-1, H_kv, d)[:len(tok)], v.view(-1, H_kv, d)[:len(tok)]
    K[0, tok.cuda()], V[0, tok.cuda()] = k.cuda(), v.cuda()
    blocks = torch.tensor(listed, dtype=torch.int32, device="cuda").expand(1, H_kv, 4).contiguous()
    case = _c(1, len(tok), H, H_kv, d, len(tok), 1, 1, causal=False)
    ref = reference(case, Q, k, v, torch.zeros(1, H_kv, 1, dtype=torch.int32))
    bound = HALF * ref["O"].abs() + (1 + HALF) * (HALF + 4 * ref["E"] + 2.0 ** -14)[..., None] * ref["O_mag"]
    O = lemo.lemo_block_attention_step(Q.cuda(), K, V, torch.tensor([S], dtype=torch.int32, device="cuda"), blocks, b)
    close("step", O, ref["O"], bound)
    O, _ = lemo.lemo_block_attention(Q.cuda(), K[0], V[0], blocks, b, 1, q_start=S - 1)
    close("prompt", O, ref["O"], bound)


@pytest.mark.gpu
def test_replayed_graphs_on_a_side_stream(lemo):
    Q, K, V, dO = (x.cuda() for x in draw(6, (300, 8, 128), (300, 2, 128), (300, 2, 128), (300, 8, 128)))
    lengths = torch.tensor([250, 300], dtype=torch.int32, device="cuda")
    cache_k, cache_v = K.expand(2, 300, 2, 128).contiguous(), V.expand(2, 300, 2, 128).contiguous()
    step_means = torch.zeros(2, 10, 2, 128, device="cuda")

    def all_of_it():
        means = lemo.lemo_block_means(K, 32)
        blocks = lemo.lemo_select_blocks(Q, means, 300, 32, 16, 4)
        O, lse2 = lemo.lemo_block_attention(Q, K, V, blocks, 32, 16)
        grads = lemo.lemo_block_attention_grad(dO, Q, K, V, O, lse2, blocks, 32, 16)
        lemo.lemo_block_means_step(cache_k, lengths, 32, step_means)
        few = lemo.lemo_select_blocks_step(Q[:2], step_means, lengths, 32, 4, S_max=300)
        return [means, blocks, O, lse2, *grads, step_means, few, lemo.lemo_block_attention_step(Q[:2], cache_k, cache_v, lengths, few, 32)]

    want = [x.clone() for x in all_of_it()]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = all_of_it()
    side.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(want, got))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = all_of_it()
    for n in range(3):
        for x in out:
            x.fill_(1)
        lengths[0] = 250 + n
        graph.replay()
        torch.cuda.synchronize()
        eager = all_of_it()
        assert all(torch.equal(x, y) for x, y in zip(eager, out))


@pytest.mark.gpu
def test_a_layer_of_them_together(lemo):
    """Norm, projections of the normed rows, choice, attention, projection, norm with gate and add: forward and back, against torch in
    64 bits on the same lists.  Every stage rounds to bf16, 2^-8 at most and 2^-9.8 of a value in the mean square; ten such roundings on
    the longest path are 1.1 % of a result's norm, and 2 % are allowed."""
    S, H, H_kv, d, C, b, bq, T = 400, 8, 2, 64, 256, 32, 16, 4
    g = torch.Generator().manual_seed(11)
    n = lambda *s, std=1.0: (torch.randn(*s, generator=g) * std).to(torch.bfloat16).cuda()  # noqa: E731
    R, gate, dR = n(S, C), n(S, C), n(S, C)
    w1, w2, w3 = (1 + n(C, std=0.1) for _ in range(3))
    Wqkv, Wo = n((H + 2 * H_kv) * d, C, std=C ** -0.5), n(C, H * d, std=(H * d) ** -0.5)
    x = R.clone()
    N, stats0 = lemo.lemo_norm_residual(None, x, w_next=w1)
    qkv = lemo.lemo_gather_gemm(N, None, Wqkv).view(S, H + 2 * H_kv, d)
    q, k, v = qkv[:, :H], qkv[:, H:H + H_kv], qkv[:, H + H_kv:]
    blocks = lemo.lemo_select_blocks(q, lemo.lemo_block_means(k, b), S, b, bq, T)
    O, lse2 = lemo.lemo_block_attention(q, k, v, blocks, b, bq)
    Y = lemo.lemo_gather_gemm(O.view(S, H * d), None, Wo)
    how = dict(gate=gate, post=lemo.NORM_RMS, w_post=w2, w_next=w3, flags=lemo.GATE_SIGMOID, block_scale=0.5)
    N2, stats = lemo.lemo_norm_residual(Y, x, **how)
    dN2 = n(S, C)
    dx = dR.clone()
    grads = lemo.lemo_norm_residual_grad(dN2, dx, x, Y, None, stats, **how)
    dO = torch.zeros(S, H * d, dtype=torch.bfloat16, device="cuda")
    lemo.lemo_gather_gemm_dx(grads.dY, Wo, dO, None)
    dqkv = torch.cat(lemo.lemo_block_attention_grad(dO.view(S, H, d), q, k, v, O, lse2, blocks, b, bq), dim=1)
    dN = torch.zeros(S, C, dtype=torch.bfloat16, device="cuda")
    lemo.lemo_gather_gemm_dx(dqkv.view(S, -1), Wqkv, dN, None)
    dW = lemo.lemo_gather_gemm_dw(dqkv.view(S, -1), N, None)
    first = lemo.lemo_norm_residual_grad(dN, dx, R, None, None, stats0, w_next=w1)

    case = _c(S, S, H, H_kv, d, b, bq, T)
    mask = allowed(case, blocks.cpu())
    r, W, v1, gg = (t.double().cpu().requires_grad_() for t in (R, Wqkv, w1, gate))
    rms = lambda t, w: t / (t.square().mean(1, keepdim=True) + 1e-5).sqrt() * w  # noqa: E731
    y = (rms(r, v1) @ W.T).view(S, -1, d)
    out = []
    for h in range(H):
        a = (y[:, h] @ y[:, H + h * H_kv // H].T / math.sqrt(d)).masked_fill(~mask[:, h * H_kv // H], -math.inf)
        out.append(torch.softmax(a, 1) @ y[:, H + H_kv + h * H_kv // H])
    y = torch.stack(out, 1).view(S, H * d) @ Wo.double().cpu().T
    new = r + 0.5 * torch.sigmoid(gg) * rms(y, w2.double().cpu())
    n2 = rms(new, w3.double().cpu())
    ((n2 * dN2.double().cpu()).sum() + (new * dR.double().cpu()).sum()).backward()
    for name, got, want in (("N", N2, n2), ("R", x, new), ("dR", dx, r.grad), ("dW", dW, W.grad), ("dgate", grads.dgate, gg.grad), ("dw", first.dw_next, v1.grad)):
        far = (got.double().cpu() - want).norm() / want.norm()
        print(name, f"{far:.2e}", flush=True)
        assert far < 0.02, name


def test_argument_errors():
    """Refused on the host, before any launch: the addresses are never touched."""
    from paper_2501_09767_amd import lemo
    lib = lemo._lib
    P = [0x100000 * (i + 1) for i in range(20)]

    def caller(fn, names, **ok):
        return lambda **kw: fn(*[dict(ok, **kw)[k] for k in names.split()])

    f = caller(lib.lemo_block_means, "K S Hkv d dt ts hs b out st", K=P[0], S=100, Hkv=2, d=64, dt=1, ts=128, hs=64, b=32, out=P[1], st=None)
    assert f(K=None) == -1 and f(out=None) == -1 and f(S=0) == -2 and f(b=0) == -2 and f(Hkv=0) == -2 and f(ts=-8) == -2 and f(dt=7) == -3
    assert f(K=P[0] + 8) == -5 and f(hs=60) == -5 and f(d=96) == -6 and f(b=48) == -6 and f(ts=1 << 22) == -6
    f = caller(lib.lemo_select_blocks, "Q S H Hkv d dt ts hs means Sk start b bq T flags out st", Q=P[0], S=100, H=4, Hkv=2, d=64, dt=1, ts=256, hs=64,
               means=P[1], Sk=1000, start=900, b=32, bq=16, T=4, flags=1, out=P[2], st=None)
    assert f(Q=None) == -1 and f(means=None) == -1 and f(out=None) == -1 and f(S=0) == -2 and f(Sk=0) == -2 and f(start=-1) == -2 and f(bq=0) == -2 and f(T=0) == -2
    assert f(flags=2) == -2 and f(H=3) == -2 and f(T=1) == -2 and f(bq=64, T=2) == -2 and f(dt=-1) == -3 and f(ts=100) == -5 and f(out=P[2] + 1) == -5
    assert f(d=32) == -6 and f(b=40) == -6 and f(Sk=32 * 16384 + 1) == -6 and f(T=5000) == -6 and f(bq=1 << 24, S=1 << 25) == -6
    n = ctypes.c_size_t()
    assert lib.lemo_block_attention_workspace_bytes(100, 1000, 4, 2, 64, 4, 32, 16, None) == -1 and lib.lemo_block_attention_workspace_bytes(100, 1000, 4, 3, 64, 4, 32, 16, ctypes.byref(n)) == -2
    assert lib.lemo_block_attention_workspace_bytes(65536, 65536, 32, 8, 128, 16, 64, 64, ctypes.byref(n)) == 0 and n.value == 0
    assert lib.lemo_block_attention_workspace_bytes(1, 32768, 32, 8, 128, 16, 64, 1, ctypes.byref(n)) == 0 and n.value > 0
    names = "Q K V S Sk H Hkv d dt qt qh kt kh vt vh blocks T b bq start scale flags O ot oh lse ws wsb st"
    ok = dict(Q=P[0], K=P[1], V=P[2], S=100, Sk=1000, H=4, Hkv=2, d=64, dt=1, qt=256, qh=64, kt=128, kh=64, vt=128, vh=64, blocks=P[3], T=16, b=32, bq=16, start=0,
              scale=0.0, flags=1, O=P[4], ot=256, oh=64, lse=P[5], ws=P[6], wsb=1 << 30, st=None)
    f = caller(lib.lemo_block_attention, names, **ok)
    for need in ("Q", "K", "V", "blocks", "O", "ws"):
        assert f(**{need: None}) == -1, need
    assert f(S=0) == -2 and f(Sk=0) == -2 and f(H=5) == -2 and f(T=0) == -2 and f(b=-32) == -2 and f(bq=0) == -2 and f(start=-5) == -2 and f(scale=math.inf) == -2 and f(flags=3) == -2
    assert f(dt=9) == -3 and f(wsb=16) == -4 and f(ws=P[6] + 64) == -5 and f(vt=132) == -5 and f(oh=60) == -5 and f(Q=P[0] + 4) == -5 and f(lse=P[5] + 2) == -5
    assert f(dt=0) == -6 and f(d=80) == -6 and f(b=33) == -6 and f(T=4097) == -6 and f(kt=1 << 22) == -6
    assert lib.lemo_block_attention_grad_workspace_bytes(100, 1000, 4, 2, 64, 4, 32, 16, ctypes.byref(n)) == 0 and n.value > 0
    assert lib.lemo_block_attention_grad_workspace_bytes(100, 32 * 16385, 4, 2, 64, 4, 32, 16, ctypes.byref(n)) == -6
    names = "dO Q K V O lse S Sk H Hkv d dt dt_ dh qt qh kt kh vt vh ot oh blocks T b bq start scale flags dQ dK dV ws wsb st"
    ok.update(dO=P[7], dt_=256, dh=64, dQ=P[8], dK=P[9], dV=P[10])
    f = caller(lib.lemo_block_attention_grad, names, **ok)
    for need in ("dO", "Q", "K", "V", "O", "lse", "blocks", "dQ", "dK", "dV", "ws"):
        assert f(**{need: None}) == -1, need
    assert f(dt=0) == -6 and f(S=1 << 24, qt=256) == -6 and f(wsb=16) == -4 and f(dQ=P[8] + 8) == -5 and f(dh=4) == -5 and f(Sk=32 * 16385) == -6 and f(flags=4) == -2
    f = caller(lib.lemo_block_means_step, "K B S Hkv d dt ss ts hs len b out st", K=P[0], B=3, S=100, Hkv=2, d=64, dt=1, ss=12800, ts=128, hs=64, len=P[1], b=32, out=P[2], st=None)
    assert f(K=None) == -1 and f(len=None) == -1 and f(out=None) == -1 and f(B=-1) == -2 and f(S=0) == -2 and f(ss=-8) == -2 and f(ss=12804) == -5 and f(b=31) == -6 and f(B=0) == 0
    f = caller(lib.lemo_select_blocks_step, "Q B H Hkv d dt ts hs means S len b T out st", Q=P[0], B=3, H=4, Hkv=2, d=64, dt=1, ts=256, hs=64, means=P[1], S=100, len=P[2], b=32,
               T=2, out=P[3], st=None)
    assert f(Q=None) == -1 and f(len=None) == -1 and f(means=None) == -1 and f(B=-2) == -2 and f(T=0) == -2 and f(S=0) == -2 and f(len=P[2] + 2) == -5 and f(d=8) == -6 and f(B=0) == 0
    f = caller(lib.lemo_block_attention_step, "Q K V B S H Hkv d dt qt qh ks kt kh vs vt vh len blocks T b scale O ot oh ws wsb st", Q=P[0], K=P[1], V=P[2], B=3, S=100, H=4,
               Hkv=2, d=64, dt=1, qt=256, qh=64, ks=12800, kt=128, kh=64, vs=12800, vt=128, vh=64, len=P[3], blocks=P[4], T=8, b=32, scale=0.0, O=P[5], ot=256, oh=64, ws=P[6],
               wsb=1 << 30, st=None)
    for need in ("Q", "K", "V", "len", "blocks", "O", "ws"):
        assert f(**{need: None}) == -1, need
    assert f(B=-1) == -2 and f(ks=-8) == -2 and f(S=0) == -2 and f(scale=math.nan) == -2 and f(dt=0) == -6 and f(wsb=4) == -4 and f(vs=12801) == -5 and f(B=0) == 0 and f(B=0, b=7) == -6


def test_binding_refuses_tensors_that_do_not_fit(lemo):
    x = torch.zeros(4, 2, 64, dtype=torch.bfloat16)
    with pytest.raises(ValueError):
        lemo.lemo_block_means(x, 32)  # not on the GPU

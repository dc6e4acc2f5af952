"""Attention over kept tokens: values near the end of what sums in binary32 hold."""
import math

import pytest
import torch

import test_block_attention as base
from test_block_attention import HALF, close, draw


@pytest.fixture(scope="module")
def lemo():
    from paper_2501_09767_amd import lemo
    return lemo


@pytest.mark.gpu
@pytest.mark.parametrize("S,H,H_kv,d,causal", [(1500, 4, 2, 128, True), (3000, 32, 32, 128, True), (2100, 16, 4, 128, False), (900, 4, 4, 64, True)])
def test_later_logits_within_the_range_of_the_reference_and_large_values(lemo, S, H, H_kv, d, causal):
    """As in test_block_attention_values.py: logits 2^94 above the first ones, values of 2^40."""
    Q, K, V = draw(S, (S, H, d), (S, H_kv, d), (S, H_kv, d))
    V = V * 2.0 ** 40
    Q[::3] = 4.0
    K *= 0.125
    K[299::300] = 94.0 / (4.0 * d / math.sqrt(d) * math.log2(math.e))
    O = lemo.lemo_kept_attention(Q.cuda(), K.cuda(), V.cuda(), None, flags=lemo.CAUSAL if causal else 0)
    some = list(range(0, S, 7)) + list(range(S - 3, S))  # (rows of the definition, for its time)
    for h in sorted({0, H // 2, H - 1}):
        g = h * H_kv // H
        case = base._c(len(some), S, 1, 1, d, S, len(some), 1, causal=False)
        q, k, v = Q[some, h:h + 1], K[:, g:g + 1], V[:, g:g + 1]
        if causal:
            x = (q[:, 0].double() @ k[:, 0].double().T / math.sqrt(d)).masked_fill(torch.arange(S) > torch.tensor(some)[:, None], -math.inf)
            P = torch.softmax(x, 1)
            E = (d + 8) * 2.0 ** -24 / math.sqrt(d) * 1.4427 * (q[:, 0].double().abs() @ k[:, 0].double().abs().T).masked_fill(x == -math.inf, 0).amax(1)
            ref = dict(O=(P @ v[:, 0].double())[:, None], O_mag=(P @ v[:, 0].double().abs())[:, None], E=E[:, None])
        else:
            ref = base.reference(case, q, k, v, torch.zeros(1, 1, 1, dtype=torch.int32))
        close("O", O[some, h:h + 1], ref["O"], HALF * ref["O"].abs() + (1 + HALF) * (HALF + 4 * ref["E"] + 2.0 ** -14)[..., None] * ref["O_mag"])

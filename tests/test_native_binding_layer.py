"""The native marshalling of the norms and of the attention over chosen blocks does what the steps in Python do, and leaves to them what
is not plain."""
import numpy as np
import pytest
import torch

from paper_2501_09767_amd import lemo

NAMES = ("norm_residual", "norm_residual_grad", "block_means", "select_blocks", "block_attention", "block_attention_grad", "select_blocks_step", "block_attention_step")


class Refusing:
    """In the place of the native module: always the long way."""
    def __getattr__(self, name):
        return lambda *a: None


def test_what_is_not_plain_is_left_to_python():
    t = torch.ones(4, 4, 64)
    for name in NAMES:
        f = getattr(lemo._native, name)
        for args in ((), (t,) * 3, (t,) * 7, (t,) * 9, (None,) * 12, (t,) * 16, (1, "x", 2.5, None)):  # (no GPU tensor among them)
            assert f(*args) is None


def calls():
    gen = torch.Generator(device="cuda").manual_seed(3)
    bf = lambda *s: torch.randn(s, generator=gen, device="cuda").bfloat16()  # noqa: E731
    M, S, C = 40, 70, 264
    kept = torch.randperm(S, generator=gen, device="cuda")[:M].sort().values.int()
    Y, R, gate, row, w = bf(M, C), bf(S, C), bf(M, C), bf(C), bf(C)
    _, stats = lemo.lemo_norm_residual(Y, R.clone(), kept, post=1, next=2)
    H, Hkv, d, b, bq, T = 8, 2, 64, 32, 16, 3
    Q, K, V, dO = bf(S, H, d), bf(S, Hkv, d), bf(S, Hkv, d), bf(S, H, d)
    means = lemo.lemo_block_means(K, b)
    blocks = lemo.lemo_select_blocks(Q, means, S, b, bq, T)
    O, lse2 = lemo.lemo_block_attention(Q, K, V, blocks, b, bq)
    cache, lengths = torch.stack([K, V]), torch.tensor([S, 33], dtype=torch.int32, device="cuda")
    step_means = torch.stack([means, means])
    few = lemo.lemo_select_blocks_step(Q[:2], step_means, lengths, b, T, S_max=S)
    new = lambda *s, dtype=torch.bfloat16: torch.zeros(s, dtype=dtype, device="cuda")  # noqa: E731

    def norm(**kw):
        r = R.clone()
        return (*lemo.lemo_norm_residual(Y, r, kept, **kw), r)

    def grad(**kw):
        r = R.clone()
        return (*lemo.lemo_norm_residual_grad(Y, r, R, Y, kept, stats, **kw), r)

    return {
        "norm": lambda: norm(gate=gate, post=1, next=2, w_post=w, b_next=row, residual_scale=0.5, flags=lemo.GATE_SIGMOID),
        "norm_given": lambda: norm(gate=row, next=0, N=None, stats=new(M, 4, dtype=torch.float32)),
        "norm_alone": lambda: lemo.lemo_norm_residual(None, R, w_next=w, N=new(S, C)),
        "grad": lambda: grad(gate=gate, post=2, next=1, w_post=w, b_post=row, w_next=w, block_scale=0.3, flags=lemo.GATE_SIGMOID),
        "grad_shared": lambda: grad(gate=row, next=2, workspace=new(1 << 22, dtype=torch.uint8)),
        "means": lambda: (lemo.lemo_block_means(K, b),),
        "select": lambda: (lemo.lemo_select_blocks(Q, means, S, b, bq, T),),
        "select_given": lambda: (lemo.lemo_select_blocks(Q, means, S, b, bq, T, 0, 5, new(*blocks.shape, dtype=torch.int32)),),
        "attention": lambda: lemo.lemo_block_attention(Q, K, V, blocks, b, bq),
        "attention_given": lambda: lemo.lemo_block_attention(Q, K, V, blocks, b, bq, 0, 0.1, 7, new(S, H + 2, d)[:, :H], new(H, S, dtype=torch.float32)),
        "attention_grad": lambda: lemo.lemo_block_attention_grad(dO, Q, K, V, O, lse2, blocks, b, bq),
        "select_step": lambda: (lemo.lemo_select_blocks_step(Q[:2], step_means, lengths, b, T, S_max=S),),
        "attention_step": lambda: (lemo.lemo_block_attention_step(Q[:2], cache, cache, lengths, few, b, O=new(2, H, d)),),
    }, dict(Q=Q, K=K, V=V, blocks=blocks, means=means, Y=Y, R=R, kept=kept, stats=stats, dO=dO, O=O, lse2=lse2)


CALLS = ["norm", "norm_given", "norm_alone", "grad", "grad_shared", "means", "select", "select_given", "attention", "attention_given", "attention_grad", "select_step",
         "attention_step"]


@pytest.mark.gpu
@pytest.mark.parametrize("name", CALLS)
def test_same_bits_either_way(monkeypatch, name):
    f = calls()[0][name]
    taken, real = [], lemo._native

    class Watching:
        def __getattr__(self, n):
            def g(*a):
                taken.append(getattr(real, n)(*a))
                return taken[-1]
            return g
    monkeypatch.setattr(lemo, "_native", Watching())
    fast = f()
    assert len(taken) == 1 and taken[0][0] == 0
    monkeypatch.setattr(lemo, "_native", Refusing())
    slow = f()
    assert len(fast) == len(slow)
    for x, y in zip(fast, slow):
        assert (x is None) == (y is None) and (x is None or torch.equal(x, y))


@pytest.mark.gpu
def test_same_refusals_either_way(monkeypatch):
    o = calls()[1]
    Q, K, V, blocks, means, Y, R, kept, stats = (o[n] for n in ("Q", "K", "V", "blocks", "means", "Y", "R", "kept", "stats"))
    bad = [lambda: lemo.lemo_block_means(K.half(), 32), lambda: lemo.lemo_block_means(K, 33), lambda: lemo.lemo_block_means(K, 0), lambda: lemo.lemo_block_means(K.transpose(1, 2), 32),
           lambda: lemo.lemo_select_blocks(Q, means, 70, 32, 64, 1), lambda: lemo.lemo_select_blocks(Q, means, 500, 32, 16, 3), lambda: lemo.lemo_select_blocks(Q, means.double(), 70, 32, 16, 3),
           lambda: lemo.lemo_block_attention(Q, K, V, blocks, 32, 8), lambda: lemo.lemo_block_attention(Q, K, V[:50], blocks, 32, 16), lambda: lemo.lemo_block_attention(Q, K, V, blocks.long(), 32, 16),
           lambda: lemo.lemo_block_attention(Q, K, V, blocks, 32, 16, 2), lambda: lemo.lemo_block_attention(Q.float(), K.float(), V.float(), blocks, 32, 16),
           lambda: lemo.lemo_block_attention_grad(o["dO"][:5], Q, K, V, o["O"], o["lse2"], blocks, 32, 16), lambda: lemo.lemo_block_attention(Q.cpu(), K, V, blocks, 32, 16),
           lambda: lemo.lemo_norm_residual(Y, R, kept[:5]), lambda: lemo.lemo_norm_residual(Y, R, kept.long()), lambda: lemo.lemo_norm_residual(Y, R, kept, next=7),
           lambda: lemo.lemo_norm_residual(Y, R, kept, w_next=Y), lambda: lemo.lemo_norm_residual(Y.float(), R, kept), lambda: lemo.lemo_norm_residual(Y[:, :260], R[:, :260], kept),
           lambda: lemo.lemo_norm_residual_grad(None, R.clone(), R, Y, kept, stats), lambda: lemo.lemo_norm_residual_grad(Y, R.clone(), R, Y, kept, stats[:4])]
    seen = []
    for native in (lemo._native, Refusing()):
        monkeypatch.setattr(lemo, "_native", native)
        seen.append([])
        for f in bad:
            with pytest.raises(Exception) as e:
                f()
            seen[-1].append((type(e.value), str(e.value)))
    assert seen[0] == seen[1]
    # values that are no plain Python numbers go the long way and do the same
    monkeypatch.undo()
    assert torch.equal(lemo.lemo_block_means(K, np.int64(32)), means)
    assert lemo.lemo_block_means(K, 32).data_ptr() != means.data_ptr()

"""The native marshalling of the rotation of queries and keys, of dropout and of the vocabulary's loss does what the steps in Python do, and leaves
to them what is not plain."""
import numpy as np
import pytest
import torch

from paper_2501_09767_amd import lemo

NAMES = ("qk_rotate", "qk_rotate_grad", "qk_rotate_step", "dropout_add", "dropout_add_grad", "vocab_loss", "vocab_loss_grad")


class Refusing:
    """In the place of the native module: always the long way."""
    def __getattr__(self, name):
        return lambda *a: None


def test_what_is_not_plain_is_left_to_python():
    t = torch.ones(4, 4, 64)
    for name in NAMES:
        f = getattr(lemo._native, name)
        for args in ((), (t,) * 3, (t,) * 6, (t,) * 11, (None,) * 13, (t,) * 14, (t,) * 15, (None,) * 17, (1, "x", 2.5, None)):  # (no GPU tensor among them)
            assert f(*args) is None


def operands():
    gen = torch.Generator(device="cuda").manual_seed(3)
    bf = lambda *s: torch.randn(s, generator=gen, device="cuda").bfloat16()  # noqa: E731
    M, S, C, H, Hkv, d, V = 40, 70, 264, 8, 2, 64, 501
    return dict(qkv=bf(M, H + 2 * Hkv, d), dQ=bf(M, H, d), dK=bf(M, Hkv, d), w=bf(d), w_q=bf(H, d), w_k=bf(Hkv, d), freq=torch.rand(16, generator=gen, device="cuda"),
                kept=torch.randperm(S, generator=gen, device="cuda")[:M].sort().values.int(), cache=bf(M, 9, Hkv, d), lengths=torch.arange(M, device="cuda", dtype=torch.int32) % 10,
                Y=bf(M, C), R=bf(S, C), rng=torch.tensor([3, 4], device="cuda"), X=bf(S, C), W=bf(V, C) / 8,
                labels=torch.randint(-1, V, (M,), generator=gen, device="cuda", dtype=torch.int32), weights=torch.rand(M, generator=gen, device="cuda"))


def calls():
    o = operands()
    Q, K, Vv = o["qkv"][:, :8], o["qkv"][:, 8:10], o["qkv"][:, 10:]
    new = lambda *s, dtype=torch.bfloat16: torch.zeros(s, dtype=dtype, device="cuda")  # noqa: E731
    head = (o["X"], o["kept"], o["W"], o["labels"])
    lse = lemo.lemo_vocab_loss(*head).lse
    how = dict(softcap=20.0, smoothing=0.1, z_weight=1e-3)

    def step(v=True, **kw):
        caches = o["cache"].clone(), o["cache"].clone() if v else None
        return (lemo.lemo_qk_rotate_step(Q, K, Vv if v else None, *caches, o["lengths"], o["freq"], **kw), *caches)

    return {
        "rotate": lambda: lemo.lemo_qk_rotate(Q, K, o["freq"], o["kept"], w_q=o["w"], w_k=o["w"]),
        "rotate_given": lambda: lemo.lemo_qk_rotate(Q, K, o["freq"], None, pos_start=-5, norm=lemo.NORM_LAYER, w_q=o["w_q"], eps=0.5, amplitude=2.0, flags=lemo.ROTATE_PAIRS,
                                                    Q_out=new(8, 40, 64).transpose(0, 1), K_out=new(40, 2, 64)),
        "rotate_one": lambda: lemo.lemo_qk_rotate(None, K, None, norm=lemo.NORM_RMS, w_k=o["w_k"]),
        "rotate_grad": lambda: lemo.lemo_qk_rotate_grad(o["dQ"], o["dK"], Q, K, o["freq"], o["kept"], w_q=o["w_q"], w_k=o["w_k"], norm=lemo.NORM_LAYER),
        "rotate_grad_given": lambda: lemo.lemo_qk_rotate_grad(o["dQ"], o["dK"], Q, K, o["freq"], w_k=o["w"], dQ=new(40, 8, 64), workspace=new(1 << 22, dtype=torch.uint8)),
        "rotate_grad_alone": lambda: lemo.lemo_qk_rotate_grad(o["dQ"], None, None, None, o["freq"], norm=lemo.NORM_NONE, weights=False),
        "step": lambda: step(w_q=o["w"], w_k=o["w"]),
        "step_keys": lambda: step(v=False, norm=lemo.NORM_NONE, Q_out=new(40, 8, 64)),
        "drop": lambda: (lemo.lemo_dropout_add(o["Y"], o["R"].clone(), o["kept"], o["rng"], 0.25, 7),),
        "drop_grad": lambda: (lemo.lemo_dropout_add_grad(o["R"], o["kept"], o["rng"], 0.25),),
        "drop_grad_given": lambda: (lemo.lemo_dropout_add_grad(o["R"], None, o["rng"], 0.25, 2, new(40, 264)),),
        "loss": lambda: lemo.lemo_vocab_loss(*head, **how),
        "loss_given": lambda: lemo.lemo_vocab_loss(*head, loss=new(40, dtype=torch.float32), lse=new(40, dtype=torch.float32), workspace=new(1 << 22, dtype=torch.uint8)),
        "loss_grad": lambda: lemo.lemo_vocab_loss_grad(o["weights"], *head, lse, **how),
        "loss_grad_given": lambda: lemo.lemo_vocab_loss_grad(o["weights"][:1], *head, lse, want_dX=False, dW=new(501, 280)[:, :264], piece=128),
    }, o


CALLS = ["rotate", "rotate_given", "rotate_one", "rotate_grad", "rotate_grad_given", "rotate_grad_alone", "step", "step_keys", "drop", "drop_grad", "drop_grad_given", "loss",
         "loss_given", "loss_grad", "loss_grad_given"]


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
    assert len(taken) == 1 and (taken[0] == 0 or taken[0][0] == 0)
    monkeypatch.setattr(lemo, "_native", Refusing())
    slow = f()
    assert len(fast) == len(slow) and type(fast) is type(slow)
    for x, y in zip(fast, slow):
        assert (x is None) == (y is None) and (x is None or torch.equal(x, y))


@pytest.mark.gpu
def test_same_refusals_either_way(monkeypatch):
    o = operands()
    Q, K, f, kept, cache, lengths, Y, R, rng, X, W, labels, w = (o["qkv"][:, :8], o["qkv"][:, 8:10], o["freq"], o["kept"], o["cache"], o["lengths"], o["Y"], o["R"], o["rng"],
                                                                 o["X"], o["W"], o["labels"], o["weights"])
    rotate, grad, step = lemo.lemo_qk_rotate, lemo.lemo_qk_rotate_grad, lemo.lemo_qk_rotate_step
    bad = [lambda: rotate(Q, K[:5], f), lambda: rotate(Q, K.float(), f), lambda: rotate(Q, K, f.double()), lambda: rotate(Q, K, f, kept[:5]), lambda: rotate(Q, K, f, kept.long()),
           lambda: rotate(Q, K, f[:7]), lambda: rotate(Q, K, o["freq"].repeat(3)), lambda: rotate(Q, K, f, norm=5), lambda: rotate(Q, K, f, norm=0, w_q=o["w"]),
           lambda: rotate(Q, K, f, w_q=o["w_q"], w_k=o["w"]), lambda: rotate(Q, K, f, w_q=o["w_k"]), lambda: rotate(Q, K, f, Q_out=K), lambda: rotate(Q, None, f, K_out=K),
           lambda: rotate(Q.half(), None, f), lambda: rotate(Q.transpose(1, 2), None, f), lambda: rotate(Q.cpu(), K, f), lambda: rotate(Q, K, f, flags=8),
           lambda: rotate(Q, K, f, pos_start=2 ** 40), lambda: rotate(Q, K, f, eps=-1.0), lambda: rotate(Q, K, f, Q_out=Q[:1].expand(40, 8, 64)),
           lambda: grad(o["dQ"], o["dK"], None, K, f), lambda: grad(o["dQ"], o["dK"], K, Q, f), lambda: grad(o["dQ"], o["dK"], Q, K, f, w_q=o["w"], workspace=torch.empty(16, device="cuda")),
           lambda: step(Q, K, None, cache, cache, lengths, f), lambda: step(Q, K, K, cache, cache[:5], lengths, f), lambda: step(Q, K, K, cache, cache, lengths[:3], f),
           lambda: step(Q, K, Q, cache, cache, lengths, f),
           lambda: lemo.lemo_dropout_add(Y, R, kept, rng, 1.0), lambda: lemo.lemo_dropout_add(Y, R, kept, rng[:1], 0.5), lambda: lemo.lemo_dropout_add(Y.float(), R, kept, rng, 0.5),
           lambda: lemo.lemo_dropout_add(Y, R, kept[:3], rng, 0.5), lambda: lemo.lemo_dropout_add_grad(R, kept, rng.float(), 0.5), lambda: lemo.lemo_dropout_add_grad(R, kept, rng, 0.5, 0, R),
           lambda: lemo.lemo_vocab_loss(X, kept, W, labels.long()), lambda: lemo.lemo_vocab_loss(X, kept[:3], W, labels), lambda: lemo.lemo_vocab_loss(X, kept, W[:, :256], labels),
           lambda: lemo.lemo_vocab_loss(X, kept, W.float(), labels), lambda: lemo.lemo_vocab_loss(X, kept, W, labels, softcap=-1.0),
           lambda: lemo.lemo_vocab_loss(X[:, :260], kept, W[:, :260], labels), lambda: lemo.lemo_vocab_loss(X, kept, W, labels, workspace=torch.empty(8, device="cuda")),
           lambda: lemo.lemo_vocab_loss_grad(w[:7], X, kept, W, labels, w), lambda: lemo.lemo_vocab_loss_grad(w, X, kept, W, labels, w[:3]),
           lambda: lemo.lemo_vocab_loss_grad(w, X, kept, W, labels, w, dX=Y[:3]), lambda: lemo.lemo_vocab_loss_grad(w, X, kept, W, labels, w, piece=-1)]
    seen = []
    for native in (lemo._native, Refusing()):
        monkeypatch.setattr(lemo, "_native", native)
        seen.append([])
        for i, g in enumerate(bad):
            with pytest.raises(Exception) as e:
                g()
                pytest.fail(f"call {i} went through")
            seen[-1].append((type(e.value), str(e.value)))
    assert seen[0] == seen[1]
    # values that are no plain Python numbers go the long way and do the same
    monkeypatch.undo()
    assert torch.equal(lemo.lemo_dropout_add_grad(R, kept, rng, np.float64(0.5), np.int64(3)), lemo.lemo_dropout_add_grad(R, kept, rng, 0.5, 3))
    assert torch.equal(lemo.lemo_dropout_add_grad(R, kept, rng, 0.5, 2 ** 64 - 1), lemo.lemo_dropout_add_grad(R, kept, rng, 0.5, -1))

"""What rounding G to bf16 leaves in the gradients of the vocabulary's loss: against the results of the formulas in 64 bits, rounded once.

A result differs from those where its error before the store, d, moves it across a boundary between two values: by a step q, for d / q of the elements, so by the root of
q |d| on the mean.  q is at most 2^-7 of a value.  d is what the roundings of G leave, each uniform within half a step, at most 2^-8 of the element, whose root mean square
is below 2^-8 / sqrt(3); they are independent, so their squares add up; and binary32 arithmetic on top: 2^-20 of the terms, and a logit's C roundings of sums no larger than
itself or a random walk's length, with 8 of lse, in the probabilities.  Which elements of G count with 2^-8:
  dX  all but the label's, whose rest it gets back
  dW  of few rows none: what rounding leaves has rows of its own, so 2^-17;  of more rows all, but for one gradient for all rows the label's is made 1, and off by
      the probability of the label alone where that is small
The bound is 1.5 times what follows (means over thousands of elements).  The roundings that these sums leave out would be 1.7e-3 of the norm and more by themselves."""
import math

import pytest
import torch


@pytest.fixture(scope="module")
def lemo():
    from paper_2501_09767_amd import lemo
    return lemo


def inputs(M, C, V, lean, seed):
    """lean: how far rows lean towards their labels' weights (0: as before any training)."""
    g = torch.Generator().manual_seed(seed)
    W = (torch.randn(V, C, generator=g) * 1.3 / math.sqrt(C)).bfloat16()
    labels = torch.randint(0, V, (M,), generator=g).int()
    X = torch.randn(M, C, generator=g)
    X += torch.rand(M, 1, generator=g) * lean * W[labels.long()].float()
    if M > 4:
        labels[3] = -100
    return X.bfloat16(), W, labels, torch.rand(M, generator=g) + 0.1


def exact(X, W, labels, w, s):
    """G, dX, dW in 64 bits, where the labels are, what binary32 leaves in G, and the probabilities."""
    X, W, w = X.double(), W.double(), w.double()
    ok = labels >= 0
    hot = torch.zeros(X.shape[0], W.shape[0], dtype=torch.float64, device=X.device)
    hot[ok, labels[ok].long()] = 1.0
    x, w = X @ W.t(), (w * ok)[:, None]
    p = torch.softmax(x, 1)
    G = (p - (1 - s) * hot - s / W.shape[0]) * w
    walk = math.sqrt(X.shape[1]) * (x.abs() + (X ** 2 @ W.t() ** 2).sqrt()) + 8 * torch.logsumexp(x, 1).abs()[:, None]
    return G, G @ W, G.t() @ X, hot, 2.0 ** -24 * walk * p * w, p


def moved(value, d2):
    """Bound of the norm of (rounded from a value off by the root of d2) - (rounded from the value)."""
    return 1.5 * (2.0 ** -7 * value.abs() * d2.sqrt()).sum().sqrt().item()


def errors(G, X, W, hot, narrow, label, rest):
    """Squares of the errors of dX and dW before their store.  G's roundings leave 2^-8 of all but the label's element in dX, `rest` times that and `label` in dW."""
    h, X, W = 2.0 ** -8 / math.sqrt(3), X.double(), W.double()
    other = (h * G * (1 - hot)) ** 2
    low = 2.0 ** -20
    dX = (other + narrow ** 2) @ W ** 2 + (low * (G.abs() @ W.abs())) ** 2
    dW = (rest ** 2 * other + label ** 2 + narrow ** 2).t() @ X ** 2 + (low * (G.abs().t() @ X.abs())) ** 2
    return dX, dW


def check(name, got, value, d2):
    off = (got.double() - value.bfloat16().double()).norm().item()
    bound = moved(value, d2)
    print(f"{name}: {off / value.norm().item():.2e} of the norm, bound {bound / value.norm().item():.2e}", flush=True)
    assert off <= bound, f"{name}: {off:.3g}, bound {bound:.3g}"


FEW = [(1, 256, 1000), (1, 1024, 4003), (2, 1024, 8000), (3, 512, 2001), (9, 136, 5000), (16, 1024, 3000), (31, 264, 1003), (31, 1024, 8000)]


@pytest.mark.gpu
@pytest.mark.parametrize("M, C, V", FEW)
def test_gradients_of_few_rows(lemo, M, C, V):
    for seed in range(6):
        X, W, labels, w = (t.cuda() for t in inputs(M, C, V, 6, 100 * M + seed))
        lse = lemo.lemo_vocab_loss(X, None, W, labels).lse
        for dloss, s, piece in ((w, 0.0, 0), (w[:1] / 3, 0.1, 0), (w, 0.1, 512)):
            G, dX, dW, hot, narrow, _ = exact(X, W, labels, dloss.expand(M), s)
            got = lemo.lemo_vocab_loss_grad(dloss, X, None, W, labels, lse, smoothing=s, piece=piece)
            eX, eW = errors(G, X, W, hot, narrow, 2.0 ** -17 * hot * G.abs(), 2.0 ** -9)
            check("dX", got[0], dX, eX)
            check("dW", got[1], dW, eW)
            assert torch.equal(lemo.lemo_vocab_loss_grad(dloss, X, None, W, labels, lse, smoothing=s, piece=piece, want_dX=False)[1], got[1])
            assert torch.equal(lemo.lemo_vocab_loss_grad(dloss, X, None, W, labels, lse, smoothing=s, piece=piece, want_dW=False)[0], got[0])


@pytest.mark.gpu
@pytest.mark.parametrize("M, C, V", [(33, 256, 3000), (300, 512, 8000), (700, 264, 2003)])
def test_the_label_in_the_gradient_of_the_rows(lemo, M, C, V):
    """Gradients of their own."""
    X, W, labels, w = (t.cuda() for t in inputs(M, C, V, 6, M))
    lse = lemo.lemo_vocab_loss(X, None, W, labels).lse
    for s in (0.0, 0.1):
        G, dX, _, hot, narrow, _ = exact(X, W, labels, w, s)
        check("dX", lemo.lemo_vocab_loss_grad(w, X, None, W, labels, lse, smoothing=s)[0], dX, errors(G, X, W, hot, narrow, 0 * hot, 1.0)[0])


@pytest.mark.gpu
@pytest.mark.parametrize("M, C, V", [(100, 256, 32000), (513, 512, 20001)])
def test_one_gradient_for_all_rows(lemo, M, C, V):
    """The mean's, as before any training: every label's element is the same, and its rounding would be in all of them."""
    X, W, labels, _ = (t.cuda() for t in inputs(M, C, V, 0, M))
    forward = lemo.lemo_vocab_loss(X, None, W, labels)
    for s in (0.0, 0.1):
        for dloss in (forward.total[3:], torch.tensor([0.37], device="cuda")):
            G, dX, dW, hot, narrow, p = exact(X, W, labels, dloss.expand(M), s)
            got = lemo.lemo_vocab_loss_grad(dloss, X, None, W, labels, forward.lse, smoothing=s)
            # the label's share: (p - s / V) / (1 - s) - 1, stored as -1 where the rest is below 2^-9
            left = hot * ((p - s / V) * dloss.double()).abs()
            assert (left <= 2.0 ** -9 * (1 - s) * dloss.double()).all()
            eX, eW = errors(G, X, W, hot, narrow, left, 1.0)
            check("dX", got[0], dX, eX)
            check("dW", got[1], dW, eW)

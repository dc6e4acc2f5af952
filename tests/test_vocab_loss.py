"""Cross entropy over a vocabulary and its gradients, against the formulas in 64 bits.

Tolerances, all as bounds that no order of the sums can pass.  With U = 2^-24 and |X||W|^T the magnitudes of a logit's terms:
  logit     C + 16 roundings of its terms (binary32 products from three bf16 parts lose 2^-24 of a product more); capped: 16 U of the result and 2 U of
            the argument on top (an exponential, a quotient and a difference against 0.3 and more, or a series)
  lse       the largest logit's error, 4 U of the largest logit and of lse itself (products with log2 e), and the sum's relative error: fewer than
            64 + V / 64 roundings
  loss      what enters it, each with its error, and 8 roundings
  G         p times the errors of its exponent, 16 roundings, and in bf16 half a step (2^-8)
  dX, dW    the sums of G's errors against the other operand's magnitudes, as many roundings as there are terms, half a step of the result"""
import ctypes
import math

import pytest
import torch

U = 2.0 ** -24


@pytest.fixture(scope="module")
def lemo():
    from paper_2501_09767_amd import lemo
    return lemo


def reference(X, W, labels, cap, s, z, w, half):
    """X [M,C] (the kept rows), W [V,C], w [M] in 64 bits -> {name: (value, bound)}; half: half a step of G's and the results' type."""
    M, C, V = X.shape[0], X.shape[1], W.shape[0]
    ok = (labels >= 0) & (labels < V)
    at = labels.long().clamp(0, V - 1)
    x, mag = X @ W.t(), X.abs() @ W.abs().t()
    e = (C + 16) * U * mag
    if cap:
        u, slope = cap * torch.tanh(x / cap), 1 - torch.tanh(x / cap) ** 2
        e = e + 16 * U * u.abs() + 2 * U * x.abs()
    else:
        u, slope = x, torch.ones_like(x)
    top, lse = u.amax(1), torch.logsumexp(u, 1)
    e_lse = e.amax(1) + 4 * U * (u.abs().amax(1) + lse.abs()) + (64 + V / 64) * U
    hit = u.gather(1, at[:, None])[:, 0]
    loss = lse - (1 - s) * hit - s * u.mean(1) + z * lse ** 2
    e_loss = e_lse * (1 + 2 * abs(z) * lse.abs()) + e.gather(1, at[:, None])[:, 0] + s * e.mean(1)
    e_loss = e_loss + 8 * U * (lse.abs() + hit.abs() + abs(z) * lse ** 2) + s * (72 + V / 64) * U * u.abs().mean(1)
    p = torch.exp(u - lse[:, None])
    hot = torch.zeros_like(u)
    hot[ok, at[ok]] = 1.0
    f = 1 + 2 * z * lse[:, None]
    parts = p * f.abs() + (1 - s) * hot + s / V
    g = (p * f - (1 - s) * hot - s / V) * slope
    e_g = p * (f.abs() * (e + e_lse[:, None] + 4 * U * (u.abs() + lse.abs()[:, None])) + 2 * abs(z) * e_lse[:, None]) + 16 * U * parts
    if cap:
        e_g = e_g * slope + parts * (2 * e / cap + 8 * U)
    w = torch.where(ok, w, 0.0)[:, None]
    g, e_g = torch.where(ok[:, None], g * w, 0.0), torch.where(ok[:, None], e_g * w.abs(), 0.0)
    stored = half if half > U else 0.0
    e_g = e_g + (stored + U) * (g.abs() + e_g)
    live = torch.where(ok[:, None], X, 0.0)
    dX, dW = g @ W, g.t() @ live
    e_dX = e_g @ W.abs() + (V + 64) * U * (g.abs() @ W.abs())
    e_dW = e_g.t() @ live.abs() + (M + 64) * U * (g.abs().t() @ live.abs())
    loss, e_loss = torch.where(ok, loss, 0.0), torch.where(ok, e_loss, 0.0)
    return dict(loss=(loss, e_loss), lse=(lse, e_lse), dX=(dX, e_dX + half * (dX.abs() + e_dX)), dW=(dW, e_dW + half * (dW.abs() + e_dW)))


def check(name, got, want):
    value, bound = want
    got = got.double().cpu()
    assert got.shape == value.shape and torch.isfinite(got).all(), name
    off = (got - value).abs() - bound
    assert off.max() <= 1e-38, f"{name}: {off.max().item():.3g} over the bound"


def inputs(dtype, M, S, C, V, kept, seed):
    g = torch.Generator().manual_seed(seed)
    W = (torch.randn(V, C, generator=g) * 2 / math.sqrt(C)).to(dtype)
    labels = torch.randint(0, V, (M,), generator=g).int()
    idx = torch.randint(0, S, (M,), generator=g).int() if kept else None  # in any order, some twice
    X = torch.randn(S, C, generator=g)
    rows = idx.long() if kept else torch.arange(M)
    X[rows] += W[labels.long()].float() * torch.rand(M, 1, generator=g) * 4
    for i, label in enumerate((-100, V, -2 ** 31, 2 ** 31 - 1, -1)):  # rows that do not count
        if M > 2 * i + 2:
            labels[2 * i + 1] = label
    if M > 12:
        labels[12], labels[11] = 0, V - 1
    return X.to(dtype), W, labels, idx, torch.randn(M, generator=g)


CASES = [  # dtype, M, S, C, V, kept, softcap, smoothing, z_weight, piece
    (torch.bfloat16, 1, 1, 8, 1, False, 0.0, 0.0, 0.0, 0),
    (torch.bfloat16, 1, 7, 64, 1000, True, 0.0, 0.0, 0.0, 0),
    (torch.bfloat16, 3, 3, 8, 7, False, 0.0, 0.1, 0.0, 0),
    (torch.bfloat16, 16, 40, 264, 3001, True, 5.0, 0.1, 1e-3, 64),
    (torch.bfloat16, 65, 65, 512, 129, False, 0.0, 0.0, 1e-2, 0),
    (torch.bfloat16, 130, 600, 128, 8193, True, 0.0, 0.2, 0.0, 1000),
    (torch.bfloat16, 300, 300, 1024, 2500, False, 30.0, 0.0, 0.0, 0),
    (torch.bfloat16, 513, 800, 72, 5000, True, 0.0, 1.0, 0.0, 2048),
    (torch.bfloat16, 2100, 2100, 64, 9000, False, 0.0, 0.0, 1e-3, 0),
    (torch.bfloat16, 1500, 4000, 256, 4096, True, 10.0, 0.1, 1e-3, 1500),
    (torch.float32, 1, 1, 4, 3, False, 0.0, 0.0, 0.0, 0),
    (torch.float32, 20, 50, 68, 1001, True, 5.0, 0.1, 1e-3, 100),
    (torch.float32, 257, 257, 256, 515, False, 0.0, 0.1, 0.0, 0),
    (torch.float32, 600, 900, 132, 2050, True, 30.0, 0.0, 1e-3, 700),
    (torch.float32, 1200, 1200, 64, 4099, False, 0.0, 0.0, 0.0, 0),
]


@pytest.mark.gpu
@pytest.mark.parametrize("case", range(len(CASES)))
def test_loss_and_gradient_against_64_bits(lemo, case):
    dtype, M, S, C, V, kept, cap, s, z, piece = CASES[case]
    print(CASES[case], flush=True)
    X, W, labels, idx, w = inputs(dtype, M, S, C, V, kept, case)
    rows = idx.long() if kept else torch.arange(M)
    want = reference(X[rows].double(), W.double(), labels, cap, s, z, w.double(), torch.finfo(dtype).eps / 2)
    c = [t.cuda() if t is not None else None for t in (X, idx, W, labels)]
    how = dict(softcap=cap, smoothing=s, z_weight=z)
    got = lemo.lemo_vocab_loss(*c, **how)
    check("loss", got.loss, want["loss"])
    check("lse", got.lse, want["lse"])
    n = int(((labels >= 0) & (labels < V)).sum())
    assert not got.loss.cpu()[(labels < 0) | (labels >= V)].any()
    total = got.loss.double().sum().item()
    for have, exact in zip(got.total.tolist(), (total, n, total / max(n, 1), 1 / n if n else 0.0)):
        assert abs(have - exact) <= 2 * U * abs(exact) + 1e-12 * got.loss.double().abs().sum().item()
    dX, dW = lemo.lemo_vocab_loss_grad(w.cuda(), *c, got.lse, piece=piece, **how)
    check("dX", dX, want["dX"])
    check("dW", dW, want["dW"])
    # one gradient for all rows; each result by itself
    one = torch.tensor([0.37], device="cuda")
    same = torch.full((M,), 0.37, device="cuda")
    both, alone = lemo.lemo_vocab_loss_grad(one, *c, got.lse, **how), lemo.lemo_vocab_loss_grad(one, *c, got.lse, want_dW=False, **how)
    shared = reference(X[rows].double(), W.double(), labels, cap, s, z, same.double().cpu(), torch.finfo(dtype).eps / 2)
    check("dX, shared", both[0], shared["dX"])
    check("dW, shared", both[1], shared["dW"])
    assert alone[1] is None and torch.equal(alone[0], both[0])
    assert torch.equal(lemo.lemo_vocab_loss_grad(one, *c, got.lse, want_dX=False, **how)[1], both[1])


@pytest.mark.gpu
def test_gradient_against_differences(lemo):
    """binary32, centred differences of the losses' sum in 64 bits; step 2^-5: truncation (h^2 / 6 of third derivatives below 1) and rounding (10 losses
    of 8 off by 2^-21 each, over h) stay below 1e-3."""
    M, C, V = 10, 16, 40
    X, W, labels, _, w = inputs(torch.float32, M, M, C, V, False, 5)
    X, W, labels, w = X.cuda(), W.cuda(), labels.cuda(), w.cuda()
    how = dict(softcap=6.0, smoothing=0.1, z_weight=0.01)
    total = lambda X, W: (lemo.lemo_vocab_loss(X, None, W, labels, **how).loss.double() * w.double()).sum().item()  # noqa: E731
    dX, dW = lemo.lemo_vocab_loss_grad(w, X, None, W, labels, lemo.lemo_vocab_loss(X, None, W, labels, **how).lse, **how)
    h = 2.0 ** -5
    for grad, name in ((dX, "X"), (dW, "W")):
        for at in range(0, grad.numel(), grad.numel() // 7):
            e = torch.zeros(grad.numel(), device="cuda")
            e[at] = h
            e = e.view_as(grad)
            slope = (total(X + e, W) - total(X - e, W)) / (2 * h) if name == "X" else (total(X, W + e) - total(X, W - e)) / (2 * h)
            assert abs(slope - grad.view(-1)[at].item()) <= 2e-3 * (1 + abs(slope)), (name, at)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_rows_in_place_strides_and_rows_that_do_not_count(lemo, dtype):
    M, S, C, V = 200, 333, 136, 1003
    X, W, labels, idx, w = (t.cuda() for t in inputs(dtype, M, S, C, V, True, 3))
    want = lemo.lemo_vocab_loss(X, idx, W, labels)
    grads = lemo.lemo_vocab_loss_grad(w, X, idx, W, labels, want.lse)
    compact = X[idx.long()].contiguous()
    got = lemo.lemo_vocab_loss(compact, None, W, labels)
    assert all(torch.equal(a, b) for a, b in zip(want, got))
    assert all(torch.equal(a, b) for a, b in zip(grads, lemo.lemo_vocab_loss_grad(w, compact, None, W, labels, want.lse)))

    def apart(x, extra):
        big = torch.full((x.shape[0], x.shape[1] + extra), 7.0, dtype=x.dtype, device="cuda")
        big[:, :x.shape[1]] = x
        return big[:, :x.shape[1]]

    X2, W2, dX, dW = apart(X, 24), apart(W, 8), apart(torch.zeros(M, C, dtype=dtype), 16), apart(torch.zeros(V, C, dtype=dtype), 40)
    got = lemo.lemo_vocab_loss(X2, idx, W2, labels)
    assert all(torch.equal(a, b) for a, b in zip(want, got))
    lemo.lemo_vocab_loss_grad(w, X2, idx, W2, labels, got.lse, dX=dX, dW=dW)
    assert torch.equal(dX, grads[0]) and torch.equal(dW, grads[1]) and (dX._base[:, C:] == 7).all() and (dW._base[:, C:] == 7).all()
    # a row that does not count may hold anything, in X and in dloss
    off = (labels < 0) | (labels >= V)
    bad, bad_w = compact.clone(), w.clone()
    bad[off] = math.nan
    bad[off.nonzero()[0]] = math.inf
    bad_w[off] = math.nan
    got = lemo.lemo_vocab_loss(bad, None, W, labels)
    assert torch.equal(got.loss, want.loss) and torch.equal(got.total, want.total) and torch.equal(got.lse[~off], want.lse[~off])
    assert all(torch.equal(a, b) for a, b in zip(grads, lemo.lemo_vocab_loss_grad(bad_w, bad, None, W, labels, got.lse)))
    # one that counts spoils its own row
    bad = compact.clone()
    bad[0, 3] = math.nan
    got = lemo.lemo_vocab_loss(bad, None, W, labels)
    assert torch.isnan(got.loss[0]) and torch.equal(got.loss[1:], want.loss[1:])
    dX, _ = lemo.lemo_vocab_loss_grad(w, bad, None, W, labels, got.lse)
    assert torch.isnan(dX[0]).all() and torch.equal(dX[1:], grads[0][1:])
    # none that counts
    none = torch.full((M,), -1, dtype=torch.int32, device="cuda")
    got = lemo.lemo_vocab_loss(X, idx, W, none)
    assert not got.loss.any() and not got.total.any() and torch.equal(got.lse, want.lse)
    assert not any(t.any() for t in lemo.lemo_vocab_loss_grad(got.total[3:], X, idx, W, none, got.lse))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_logits_far_apart(lemo, dtype):
    """Logits of +-1e4 (all exact): the softmax is one of its largest, whatever the piece or tile it lies in."""
    C, V = 8, 700
    X = torch.zeros(4, C)
    X[:, 0] = torch.tensor([1.0, -1.0, 64.0, 0.0])
    W = torch.zeros(V, C)
    W[:, 0] = -128.0
    W[699, 0], W[5, 0] = 128.0, 96.0
    labels = torch.tensor([699, 0, 5, 7], dtype=torch.int32)
    c = (X.to(dtype).cuda(), None, W.to(dtype).cuda(), labels.cuda())
    got = lemo.lemo_vocab_loss(*c)
    want = torch.tensor([0.0, math.log(698), 64.0 * 32, math.log(V)], dtype=torch.float64)
    assert ((got.loss.double().cpu() - want).abs() <= 2.0 ** -20 * (1 + want)).all()
    dX, dW = lemo.lemo_vocab_loss_grad(torch.ones(4, device="cuda"), *c, got.lse, piece=64)
    # row 0 in 64 bits: (96 - 128) / (1 + e^32) = -4e-13.  binary32 holds 1 / (1 + e^-32) as 1 or a step below, so the label's 128 may be missing or there
    # 2^-23 times over: 2^-16 bounds that.
    assert torch.isfinite(dX).all() and torch.isfinite(dW).all() and dX[0].abs().max().item() <= 2.0 ** -16 and dX[2, 0].item() == 32.0


@pytest.mark.gpu
@pytest.mark.parametrize("kept", [False, True])
def test_more_rows_than_a_launch_takes(lemo, kept):
    M, C, V = 33001, 8, 90
    X, W, labels, idx, w = inputs(torch.bfloat16, M, M + 5, C, V, kept, 6)
    rows = idx.long() if kept else torch.arange(M)
    want = reference(X[rows].double(), W.double(), labels, 0.0, 0.1, 0.0, w.double(), 2.0 ** -8)
    c = [t.cuda() if t is not None else None for t in (X, idx, W, labels)]
    got = lemo.lemo_vocab_loss(*c, smoothing=0.1)
    check("loss", got.loss, want["loss"])
    check("lse", got.lse, want["lse"])
    dX, dW = lemo.lemo_vocab_loss_grad(w.cuda(), *c, got.lse, smoothing=0.1)
    check("dX", dX, want["dX"])
    check("dW", dW, want["dW"])


@pytest.mark.gpu
@pytest.mark.parametrize("case", [  # M, C, V, kept, softcap, smoothing: rows of tiles in groups of 4, 2 and 1; one slab, odd numbers of slabs, a partial one; a last column tile cut short
    (1700, 136, 11000, True, 5.0, 0.1), (900, 8, 33001, False, 0.0, 0.0), (1000, 1536, 32001, True, 0.0, 0.2), (300, 64, 40000, False, 0.0, 0.0), (2305, 264, 9999, True, 0.0, 0.0),
    (256, 192, 70000, False, 30.0, 0.0)])
def test_runs_of_tiles(lemo, case):
    """More tiles of 256 x 256 than CUs, rows of up to 1536 columns: workgroups go from tile to tile."""
    print(case, flush=True)
    M, C, V, kept, cap, s = case
    X, W, labels, idx, w = (t.cuda() if t is not None else None for t in inputs(torch.bfloat16, M, M + 50, C, V, kept, 21))
    labels[-3:] = torch.tensor([0, V - 1, V // 256 * 256], dtype=torch.int32)
    want = reference((X[idx.long()] if kept else X[:M]).double(), W.double(), labels, cap, s, 1e-3, w.double(), 2.0 ** -8)
    want = {name: (value.cpu(), bound.cpu()) for name, (value, bound) in want.items()}
    got = lemo.lemo_vocab_loss(X, idx, W, labels, softcap=cap, smoothing=s, z_weight=1e-3)
    check("loss", got.loss, want["loss"])
    check("lse", got.lse, want["lse"])
    dX, dW = lemo.lemo_vocab_loss_grad(w, X, idx, W, labels, got.lse, softcap=cap, smoothing=s, z_weight=1e-3)
    check("dX", dX, want["dX"])
    check("dW", dW, want["dW"])
    again = lemo.lemo_vocab_loss(X, idx, W, labels, softcap=cap, smoothing=s, z_weight=1e-3)
    assert torch.equal(again.loss, got.loss) and torch.equal(again.lse, got.lse)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_the_largest_vocabulary_and_offsets_past_32_bits(lemo, dtype):
    """V = 2^21 rows of W (and dW) 4 KB or more apart: past 4 GiB."""
    M, C, V, ld = 3, 8, 2 ** 21, 2056
    g = torch.Generator(device="cuda").manual_seed(1)
    W, dW = (torch.empty(V, ld, dtype=dtype, device="cuda")[:, :C] for _ in range(2))
    W.copy_(torch.randn(V, C, generator=g, device="cuda"))
    dW.fill_(7)
    X = torch.randn(M, C, generator=g, device="cuda").to(dtype)
    labels = torch.tensor([V - 1, 0, V // 2 + 1], dtype=torch.int32, device="cuda")
    got = lemo.lemo_vocab_loss(X, None, W, labels)
    dX, _ = lemo.lemo_vocab_loss_grad(torch.ones(M, device="cuda"), X, None, W, labels, got.lse, dW=dW)
    x, Wd = X.double() @ W.double().t(), W.double()
    # (sums of 2^21 terms in parts of at most 2^12: 2^13 roundings; G's in bf16 off by 2^-8 each)
    lse = torch.logsumexp(x, 1)
    want = lse - x.gather(1, labels.long()[:, None])[:, 0]
    assert ((got.loss.double() - want).abs() <= 2.0 ** -11 * want).all()
    p = torch.exp(x - lse[:, None])
    p[torch.arange(M), labels.long()] -= 1
    half = torch.finfo(dtype).eps / 2
    assert ((dX.double() - p @ Wd).abs() <= (2.0 ** -11 + 2 * half) * (p.abs() @ Wd.abs())).all()
    wide = p.t() @ X.double()
    assert ((dW.double() - wide).abs() <= (2.0 ** -11 + 2 * half) * (p.abs().t() @ X.double().abs()) + 1e-30).all()


@pytest.mark.gpu
def test_no_rows_and_one_row(lemo):
    C, V = 64, 100
    W = torch.randn(V, C, device="cuda").bfloat16()
    none, labels = torch.empty(0, C, dtype=torch.bfloat16, device="cuda"), torch.empty(0, dtype=torch.int32, device="cuda")
    for X, idx in ((none, None), (W, labels)):
        got = lemo.lemo_vocab_loss(X, idx, W, labels)
        assert got.loss.shape == (0,) and not got.total.any()
        dW = torch.full((V, C), 3.0, dtype=torch.bfloat16, device="cuda")
        dX, _ = lemo.lemo_vocab_loss_grad(got.total[3:], X, idx, W, labels, got.lse, dW=dW)
        assert dX.shape == (0, C) and not dW.any()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_replayed_graphs_other_streams_and_the_same_bits(lemo, dtype):
    M, C, V = 300, 256, 2003
    X, W, labels, idx, _ = (t.cuda() for t in inputs(dtype, M, 500, C, V, True, 8))

    def step():
        got = lemo.lemo_vocab_loss(X, idx, W, labels, z_weight=1e-3)
        return [*got, *lemo.lemo_vocab_loss_grad(got.total[3:], X, idx, W, labels, got.lse, z_weight=1e-3, piece=640)]

    want = [t.clone() for t in step()]
    assert all(torch.equal(a, b) for a, b in zip(want, step()))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = step()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, got))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step()
    other = torch.randint(0, V, (M,), dtype=torch.int32, device="cuda")
    first = labels.clone()
    for chosen in (first, other, first):  # labels are read at each replay
        labels.copy_(chosen)
        eager = step()
        for t in out:
            t.fill_(3.0)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(eager, out))


def test_argument_errors():
    """Refused on the host, before any launch: the addresses are never touched."""
    from paper_2501_09767_amd import lemo
    lib = lemo._lib
    P = [0x10000 * (i + 1) for i in range(16)]
    n = ctypes.c_size_t()
    need = lib.lemo_vocab_loss_workspace_bytes
    assert need(10, 64, 100, 1, ctypes.byref(n)) == 0 and n.value > 0 and need(10, 64, 100, 1, None) == -1 and need(10, 64, 100, 2, ctypes.byref(n)) == -3
    assert need(-1, 64, 100, 1, ctypes.byref(n)) == -2 and need(1, 60, 100, 1, ctypes.byref(n)) == -6 and need(1, 64, 2 ** 21 + 1, 1, ctypes.byref(n)) == -6
    assert need(2 ** 22 + 1, 64, 100, 1, ctypes.byref(n)) == -6 and need(1, 64, 0, 1, ctypes.byref(n)) == -2
    names = "X S ldx idx M W ldw C V dt labels cap s z loss lse total ws wsb stream".split()
    ok = dict(X=P[0], S=100, ldx=64, idx=P[1], M=10, W=P[2], ldw=64, C=64, V=1000, dt=1, labels=P[3], cap=0.0, s=0.0, z=0.0, loss=P[4], lse=P[5], total=P[6], ws=P[7],
              wsb=1 << 24, stream=None)
    f = lambda **kw: lib.lemo_vocab_loss(*[dict(ok, **kw)[k] for k in names])  # noqa: E731
    assert f(dt=7) == -3 and f(X=None) == -1 and f(W=None) == -1 and f(labels=None) == -1 and f(loss=None) == -1 and f(lse=None) == -1 and f(ws=None) == -1
    assert f(cap=-1.0) == -2 and f(cap=math.inf) == -2 and f(cap=1e-40) == -2 and f(s=-0.1) == -2 and f(s=1.5) == -2 and f(s=math.nan) == -2 and f(z=math.nan) == -2
    assert f(S=0) == -2 and f(M=-1) == -2 and f(idx=None, M=101) == -2 and f(ldx=56) == -2 and f(ldw=32) == -2 and f(V=0) == -2
    assert f(C=60) == -6 and f(ldx=2 ** 22) == -6 and f(S=2 ** 25) == -6 and f(V=2 ** 21 + 1) == -6 and f(C=65544, ldx=65544, ldw=65544) == -6
    assert f(X=P[0] + 8) == -5 and f(W=P[2] + 2) == -5 and f(ldx=68) == -5 and f(labels=P[3] + 2) == -5 and f(total=P[6] + 1) == -5 and f(ws=P[7] + 16) == -5
    assert f(wsb=64) == -4
    need = lib.lemo_vocab_loss_grad_workspace_bytes
    assert need(10, 64, 100, 64, 1, 0, ctypes.byref(n)) == 0 and n.value > 0 and need(10, 64, 100, 64, 1, 0, None) == -1
    assert need(10, 64, 100, 32, 1, 0, ctypes.byref(n)) == -2 and need(10, 64, 100, 64, 1, -1, ctypes.byref(n)) == -2 and need(10, 60, 100, 64, 1, 0, ctypes.byref(n)) == -6
    small, large = ctypes.c_size_t(), ctypes.c_size_t()
    assert need(4096, 4096, 131072, 4096, 1, 1024, ctypes.byref(small)) == 0 and need(4096, 4096, 131072, 4096, 1, 131072, ctypes.byref(large)) == 0
    assert small.value < 4096 * 131072 // 2 < 4096 * 131072 * 2 <= large.value
    names = "dl dls X S ldx idx M W ldw C V dt labels lse cap s z dX lddx dW lddw piece ws wsb stream".split()
    ok = dict(ok, dl=P[8], dls=1, dX=P[9], lddx=64, dW=P[10], lddw=64, piece=0)
    f = lambda **kw: lib.lemo_vocab_loss_grad(*[dict(ok, **kw)[k] for k in names])  # noqa: E731
    assert f(dt=2) == -3 and f(dl=None) == -1 and f(lse=None) == -1 and f(ws=None) == -1 and f(X=None) == -1
    assert f(dls=2) == -2 and f(piece=-5) == -2 and f(lddx=32) == -2 and f(lddw=8) == -2 and f(s=2.0) == -2
    assert f(dX=P[9] + 8) == -5 and f(lddw=68) == -5 and f(dl=P[8] + 2) == -5 and f(lddw=2 ** 22) == -6 and f(wsb=64) == -4


def test_binding_refuses_tensors_that_do_not_fit(lemo):
    with pytest.raises(ValueError):
        lemo.lemo_vocab_loss(torch.zeros(2, 8), None, torch.zeros(3, 8), torch.zeros(2, dtype=torch.int32))  # not on the GPU

"""Dropout into the residual rows and its gradient, against the generator in Python's integers and the add in 64 bits.

Tolerance: which elements stay is exact.  A result is off by at most half a step of its type and three roundings of 2^-24 (the scale, its product,
the add) of the terms' magnitudes."""
import math

import pytest
import torch

U = 2.0 ** -24
LOW = 0xffffffff


@pytest.fixture(scope="module")
def lemo():
    from paper_2501_09767_amd import lemo
    return lemo


def philox(counter, key):
    x, k = list(counter), list(key)
    for _ in range(10):
        p, q = x[0] * 0xD2511F53, x[2] * 0xCD9E8D57
        x = [(q >> 32) ^ x[1] ^ k[0], q & LOW, (p >> 32) ^ x[3] ^ k[1], p & LOW]
        k = [(k[0] + 0x9E3779B9) & LOW, (k[1] + 0xBB67AE85) & LOW]
    return x


def keep16(p):
    return max(1, math.floor((1 - p) * 65536 + 0.5))


def mask(tokens, C, p, seed, stream):
    seed, stream = seed % 2 ** 64, stream % 2 ** 64
    out = torch.zeros(len(tokens), C, dtype=torch.bool)
    for i, k in enumerate(tokens):
        for b in range(-(-C // 8)):
            x = philox((b, k, stream & LOW, stream >> 32), (seed & LOW, seed >> 32))
            for c in range(8 * b, min(C, 8 * b + 8)):
                out[i, c] = (x[c % 8 // 2] >> (16 * (c % 2)) & 0xffff) < keep16(p)
    return out


def test_generator_known_answers():
    """The published test vectors of Philox 4x32-10 (zeros, and all bits set)."""
    assert philox((0, 0, 0, 0), (0, 0)) == [0x6627E8D5, 0xE169C58D, 0xBC57AC4C, 0x9B00DBD8]
    assert philox((LOW,) * 4, (LOW, LOW)) == [0x408F276D, 0x41C83B0E, 0xA20BC7C6, 0x6D5451FD]


CASES = [  # dtype, M, S, C, kept, p, seed, stream, site
    (torch.bfloat16, 1, 1, 8, False, 0.5, 0, 0, 0),
    (torch.bfloat16, 3, 9, 72, True, 0.1, -1, 2 ** 63 - 1, 7),
    (torch.bfloat16, 20, 20, 264, False, 0.9, 1234567890123, -5, 2 ** 64 - 1),
    (torch.bfloat16, 5, 2 ** 17, 2056, True, 0.3, 42, 1, 3),
    (torch.float32, 7, 7, 4, False, 0.25, 9, 9, 9),
    (torch.float32, 11, 40, 36, True, 0.0, 5, 6, 7),
    (torch.float32, 2, 3, 4100, True, 1 - 2 ** -20, 5, 6, 7),
    (torch.float32, 33, 50, 132, True, 2 ** -20, 3, 2, 1),
]


@pytest.mark.gpu
@pytest.mark.parametrize("case", range(len(CASES)))
def test_against_64_bits(lemo, case):
    dtype, M, S, C, kept, p, seed, stream, site = CASES[case]
    print(CASES[case], flush=True)
    g = torch.Generator().manual_seed(case)
    idx = torch.randperm(S, generator=g)[:M].to(torch.int32) if kept else None
    if kept and M > 2:
        idx[1] = (-1, S, 2 ** 31 - 1, -2 ** 31)[case % 4]  # dropped
    tokens = [i for i in range(M)] if idx is None else idx.tolist()
    there = torch.tensor([0 <= k < S for k in tokens])
    Y, R = torch.randn(M, C, generator=g).to(dtype), torch.randn(S, C, generator=g).to(dtype)
    keep = mask([k if ok else 0 for k, ok in zip(tokens, there.tolist())], C, p, seed, stream + site)
    rng = torch.tensor([seed, stream], dtype=torch.int64, device="cuda")
    ci = None if idx is None else idx.cuda()
    want, size = R.double(), torch.zeros(S, C, dtype=torch.float64)
    live = torch.tensor(tokens)[there]
    add = torch.where(keep, Y.double() * 65536 / keep16(p), 0.0)[there]
    want[live] += add
    size[live] = R.double().abs()[live] + add.abs()
    half = torch.finfo(dtype).eps / 2
    got = lemo.lemo_dropout_add(Y.cuda(), R.cuda(), ci, rng, p, site).cpu()
    off = (got.double() - want).abs() - half * want.abs() - 3 * U * size
    assert off.max() <= 0
    rest = torch.ones(S, dtype=torch.bool)
    rest[live] = False
    assert torch.equal(got[rest], R[rest])
    assert torch.equal(got[live][~keep[there]], R[live][~keep[there]])
    back = lemo.lemo_dropout_add_grad(R.cuda(), ci, rng, p, site).cpu()
    wide = torch.zeros(M, C, dtype=torch.float64)
    wide[there] = torch.where(keep[there], R.double()[live] * 65536 / keep16(p), 0.0)
    assert ((back.double() - wide).abs() - (half + 3 * U) * wide.abs()).max() <= 0
    assert not back[there][~keep[there]].any() and not back[~there].any()


@pytest.mark.gpu
def test_strides_dropped_values_and_plain_dropout_in_place(lemo):
    M, S, C, p = 50, 70, 520, 0.4
    g = torch.Generator().manual_seed(1)
    Y, R = torch.randn(M, C, generator=g).bfloat16().cuda(), torch.randn(S, C, generator=g).bfloat16().cuda()
    idx = torch.randperm(S, generator=g)[:M].to(torch.int32).cuda()
    rng = torch.tensor([77, 88], device="cuda")
    want = lemo.lemo_dropout_add(Y, R.clone(), idx, rng, p)
    keep = mask(idx.tolist(), C, p, 77, 88).cuda()
    wide = [torch.full((n, C + 24), 7.0, dtype=torch.bfloat16, device="cuda") for n in (M, S)]
    wide[0][:, :C], wide[1][:, :C] = Y, R
    wide[0][:, :C][~keep] = math.nan  # what is dropped may be anything
    assert torch.equal(lemo.lemo_dropout_add(wide[0][:, :C], wide[1][:, :C], idx, rng, p), want)
    assert (wide[0][:, C:] == 7).all() and (wide[1][:, C:] == 7).all()
    # the mask goes by the token: whatever the order and the number of the kept rows
    back = lemo.lemo_dropout_add_grad(R, idx, rng, p)
    order = torch.randperm(M, generator=g).cuda()[:20]
    assert torch.equal(lemo.lemo_dropout_add_grad(R, idx[order].contiguous(), rng, p), back[order])
    plain = lemo.lemo_dropout_add_grad(R, None, rng, p)
    assert torch.equal(plain[idx.long()], back)
    rows = R.clone()
    assert lemo.lemo_dropout_add_grad(rows, None, rng, p, dY=rows) is rows and torch.equal(rows, plain)
    # other steps and other places of a step are other masks
    assert torch.equal(lemo.lemo_dropout_add_grad(R, None, torch.tensor([77, 80], device="cuda"), p, 8), plain)
    for other, site in (([77, 88], 1), ([78, 88], 0), ([77, 88 + 2 ** 32], 0), ([77 + 2 ** 32, 88], 0)):
        assert not torch.equal(lemo.lemo_dropout_add_grad(R, None, torch.tensor(other, device="cuda"), p, site), plain)
    # no rows
    none = torch.empty(0, C, dtype=torch.bfloat16, device="cuda")
    before = R.clone()
    assert torch.equal(lemo.lemo_dropout_add(none, R, idx[:0].contiguous(), rng, p), before) and lemo.lemo_dropout_add_grad(R, idx[:0].contiguous(), rng, p).shape == (0, C)


@pytest.mark.gpu
def test_share_that_stays_and_neighbours(lemo):
    """Of n draws of probability q, n q stay within 6 deviations (one run in 5e8 would not), and neighbouring columns, rows and steps agree as often as
    independent ones."""
    S, C = 1024, 2048
    ones = torch.ones(S, C, device="cuda")
    for p in (0.1, 0.5, 0.77):
        a, b = ((lemo.lemo_dropout_add_grad(ones, None, torch.tensor([5, n], device="cuda"), p) > 0).double() for n in (1, 2))
        q = keep16(p) / 65536
        for n, k in ((a.numel(), a.sum()), (a[:, 1:].numel(), (a[:, 1:] == a[:, :-1]).sum()), (a[1:].numel(), (a[1:] == a[:-1]).sum()), (a.numel(), (a == b).sum())):
            share = q if k is not None and n == a.numel() and torch.equal(k, a.sum()) else q * q + (1 - q) * (1 - q)
            # (agreements of neighbours share draws: their variance is at most three times that of independent ones)
            assert abs(k.item() - n * share) <= 6 * math.sqrt(3 * n * share * (1 - share)), (p, n, k.item() / n, share)


@pytest.mark.gpu
def test_replayed_graphs_take_the_generator_as_it_stands(lemo):
    M, C, p = 300, 768, 0.2
    Y, R = torch.randn(M, C, device="cuda"), torch.zeros(M, C, device="cuda")
    rng = torch.tensor([1, 0], device="cuda")
    lemo.lemo_dropout_add(Y, R, None, rng, p)  # (no launch limits to raise; the first call may as well be outside)
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        other = lemo.lemo_dropout_add(Y, torch.zeros_like(Y), None, rng, p)
    torch.cuda.synchronize()
    assert torch.equal(other, R)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        lemo.lemo_dropout_add(Y, R, None, rng, p, 3)
        back = lemo.lemo_dropout_add_grad(Y, None, rng, p, 3)
        rng[1] += 16
    for step in range(4):
        R.zero_()
        back.fill_(3.0)
        now = torch.tensor([1, 16 * step], device="cuda")
        want = lemo.lemo_dropout_add(Y, torch.zeros_like(Y), None, now, p, 3)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(R, want) and torch.equal(back, want) and rng[1].item() == 16 * (step + 1)


def test_argument_errors():
    """Refused on the host, before any launch: the addresses are never touched."""
    from paper_2501_09767_amd import lemo
    lib = lemo._lib
    P = [0x10000 * (i + 1) for i in range(6)]
    names = "Y ldy R ldr S idx M p rng site C dt stream".split()
    ok = dict(Y=P[0], ldy=64, R=P[1], ldr=64, S=100, idx=P[2], M=10, p=0.5, rng=P[3], site=0, C=64, dt=1, stream=None)
    f = lambda **kw: lib.lemo_dropout_add(*[dict(ok, **kw)[k] for k in names])  # noqa: E731
    g = lambda **kw: lib.lemo_dropout_add_grad(*[dict(ok, **kw)[k] for k in "R ldr S idx M p rng site Y ldy C dt stream".split()])  # noqa: E731
    for h in (f, g):
        assert h(dt=2) == -3 and h(Y=None) == -1 and h(R=None) == -1 and h(rng=None) == -1
        assert h(p=1.0) == -2 and h(p=-0.1) == -2 and h(p=math.nan) == -2 and h(S=0) == -2 and h(M=101) == -2 and h(M=-1) == -2 and h(C=0) == -2 and h(ldy=56) == -2 and h(ldr=32) == -2
        assert h(C=60) == -6 and h(dt=0, C=62) == -6
        assert h(Y=P[0] + 8) == -5 and h(ldr=68) == -5 and h(idx=P[2] + 2) == -5 and h(rng=P[3] + 4) == -5
        assert h(M=0) == 0


def test_binding_refuses_tensors_that_do_not_fit(lemo):
    with pytest.raises(ValueError):
        lemo.lemo_dropout_add(torch.zeros(2, 8), torch.zeros(2, 8), None, torch.zeros(2, dtype=torch.int64), 0.5)  # not on the GPU

"""Norms before and after a block with its gate, its scaled add into the residual rows, and their gradients, against the formulas in
64 bits.

Tolerances: a stored value is off by at most half a step of its type (eps / 2 of it) and by the binary32 arithmetic before it: every
term that enters a result passes through fewer than 64 roundings of 2^-24 (products, two norms' sums over registers, an exponential),
so 64 * 2^-24 of the terms' magnitudes bounds it.  Sums over M rows add (rows per workgroup + parts per wave + 8) roundings."""
import ctypes
import math

import pytest
import torch

U = 2.0 ** -24


@pytest.fixture(scope="module")
def lemo():
    from paper_2501_09767_amd import lemo
    return lemo


def norm64(x, mode, w, b, eps):
    """Value, mean, 1 / deviation, magnitude of what entered."""
    if mode == 0:
        z = torch.zeros(len(x), 1, dtype=torch.float64)
        return x, z, z, x.abs()
    mean = x.mean(1, keepdim=True) if mode == 2 else torch.zeros(len(x), 1, dtype=torch.float64)
    rstd = ((x - mean).square().mean(1, keepdim=True) + eps).rsqrt()
    w = torch.ones(x.shape[1], dtype=torch.float64) if w is None else w
    b = torch.zeros_like(w) if b is None else b
    return (x - mean) * rstd * w + b, mean, rstd, (x.abs() + mean.abs()) * rstd * w.abs() + b.abs()


def back64(dy, x, mean, rstd, mode, w):
    """Gradients of a norm's input, weight, bias, and the magnitudes of the three."""
    if mode == 0:
        return dy, None, None, dy.abs(), None, None
    xh = (x - mean) * rstd
    xm = (x.abs() + mean.abs()) * rstd  # xh is a difference
    t = dy if w is None else dy * w
    c0 = t.mean(1, keepdim=True) if mode == 2 else 0.0
    dx = rstd * (t - xh * (t * xh).mean(1, keepdim=True) - c0)
    mag = rstd * (t.abs() + xm * (t.abs() * xm).mean(1, keepdim=True) + t.abs().mean(1, keepdim=True))
    return dx, (dy * xh).sum(0), dy.sum(0), mag, (dy.abs() * xm).sum(0), dy.abs().sum(0)


def inputs(dtype, M, S, C, post, nxt, gate, rows, seed):
    g = torch.Generator().manual_seed(seed)
    n = lambda *s, std=1.0: (torch.randn(*s, generator=g) * std).to(dtype)  # noqa: E731
    idx = None
    if rows == "kept":
        idx = torch.randperm(S, generator=g)[:M].to(torch.int32)
    elif rows == "dropped":
        idx = torch.randperm(S, generator=g)[:M].to(torch.int32)
        idx[::3] = torch.tensor([-1, S, 2 ** 31 - 1, -2 ** 31], dtype=torch.int32)[torch.arange(len(idx[::3])) % 4]
    t = dict(Y=n(M, C) + 0.5, R=n(S, C, std=2.0), dN=n(M, C, std=0.3), dR=n(S, C, std=0.3), idx=idx,
             gate={"none": None, "row": n(C), "rows": n(M, C), "sigmoid": n(M, C)}[gate],
             w_post=(1 + n(C, std=0.2)).to(dtype) if post else None, b_post=n(C) if post == 2 else None,
             w_next=(1 + n(C, std=0.2)).to(dtype) if nxt else None, b_next=n(C) if nxt == 2 else None)
    return t


def check(name, got, want, mag, dtype, roundings=64):
    half = torch.finfo(dtype).eps / 2
    got = got.double().cpu()
    off = (got - want).abs() - (half * want.abs() + roundings * U * (1 + half) * mag)
    assert got.shape == want.shape and torch.isfinite(got).all(), name
    assert off.numel() == 0 or off.max() <= 1e-38, f"{name}: {off.max().item():.3g} over the bound, at {divmod(int(off.argmax()), off.shape[-1])}"


SHAPES = [  # dtype, M, S, C, post, next, gate, rows
    (torch.bfloat16, 1, 1, 8, 1, 1, "rows", None),
    (torch.bfloat16, 5, 9, 264, 2, 1, "row", "kept"),
    (torch.bfloat16, 37, 64, 512, 1, 2, "sigmoid", "dropped"),
    (torch.bfloat16, 700, 700, 1024, 0, 1, "none", None),
    (torch.bfloat16, 64, 100, 2056, 1, 1, "rows", "kept"),
    (torch.bfloat16, 600, 1200, 4096, 2, 2, "sigmoid", "kept"),
    (torch.bfloat16, 30, 30, 8200, 1, 1, "row", "dropped"),
    (torch.bfloat16, 3, 4, 16384, 2, 2, "rows", "kept"),
    (torch.float32, 1, 3, 4, 2, 2, "row", "kept"),
    (torch.float32, 90, 90, 260, 1, 1, "sigmoid", None),
    (torch.float32, 33, 70, 1028, 0, 2, "rows", "dropped"),
    (torch.float32, 40, 41, 4096, 1, 0, "none", "kept"),
    (torch.float32, 21, 21, 5120, 2, 1, "rows", "kept"),
    (torch.float32, 6, 6, 16384, 1, 2, "sigmoid", "kept"),
    (torch.float32, 9, 9, 8, 2, 2, "none", None),
    (torch.bfloat16, 9, 20, 72, 2, 2, "sigmoid", "kept"),
    (torch.bfloat16, 4500, 5000, 512, 1, 2, "rows", "kept"),
    (torch.bfloat16, 2100, 2100, 2048, 2, 1, "sigmoid", None),
    (torch.float32, 4100, 4200, 132, 2, 2, "row", "dropped"),
]


@pytest.mark.gpu
@pytest.mark.parametrize("case", range(len(SHAPES)))
def test_forward_and_gradient_against_64_bits(lemo, case):
    dtype, M, S, C, post, nxt, gate, rows = SHAPES[case]
    print(SHAPES[case], flush=True)
    a, beta, eps = 0.8, -0.35, 1e-5
    t = inputs(dtype, M, S, C, post, nxt, gate, rows, seed=case)
    d = {k: v.cuda() if v is not None else None for k, v in t.items()}
    w = {k: v.double() if v is not None and v.dtype != torch.int32 else None for k, v in t.items()}
    keep = torch.arange(M) if t["idx"] is None else t["idx"].long()
    there = (keep >= 0) & (keep < S)
    live = keep[there]
    flags = lemo.GATE_SIGMOID if gate == "sigmoid" else 0
    how = dict(gate=d["gate"], post=post, next=nxt, w_post=d["w_post"], b_post=d["b_post"], w_next=d["w_next"], residual_scale=a, block_scale=beta, flags=flags)

    R = d["R"].clone()
    N, stats = lemo.lemo_norm_residual(d["Y"], R, d["idx"], b_next=d["b_next"], eps=eps, **how)
    u, mean_p, rstd_p, mag_u = norm64(w["Y"], post, w["w_post"], w["b_post"], eps)
    g = torch.ones(1, dtype=torch.float64) if gate == "none" else torch.sigmoid(w["gate"]) if gate == "sigmoid" else w["gate"]
    g = g.expand(M, C) if g.dim() == 1 else g
    r = a * w["R"][live] + beta * (g * u)[there]
    want = w["R"].clone()
    want[live] = r
    mag = torch.zeros(S, C, dtype=torch.float64)
    mag[live] = (a * w["R"][live]).abs() + abs(beta) * (g.abs() * mag_u)[there]
    check("R", R, want, mag, dtype)
    rest = torch.ones(S, dtype=torch.bool)
    rest[live] = False
    assert torch.equal(R.cpu()[rest], t["R"][rest])
    stored = R.cpu().double()[live]
    n, mean_n, rstd_n, mag_n = norm64(stored, nxt, w["w_next"], w["b_next"], eps)
    full = torch.zeros(M, 4, dtype=torch.float64)
    full[there] = torch.cat([mean_p[there], rstd_p[there], mean_n, rstd_n], 1)
    size = torch.zeros(M, 4, dtype=torch.float64)
    size[there] = torch.cat([w["Y"][there].abs().mean(1, keepdim=True), rstd_p[there] * 4, stored.abs().mean(1, keepdim=True), rstd_n * 4], 1)
    check("stats", stats, full, size, torch.float32)
    if nxt:
        wide = torch.zeros(M, C, dtype=torch.float64)
        wide[there], mag = n, torch.zeros(M, C, dtype=torch.float64)
        mag[there] = mag_n
        check("N", N, wide, mag, dtype)
    else:
        assert N is None

    dR = d["dR"].clone()
    got = lemo.lemo_norm_residual_grad(d["dN"] if nxt else None, dR, R, d["Y"], d["idx"], stats, **how)
    s64 = stats.double().cpu()
    dx, dw, db, mag_x, mag_w, mag_b = back64(w["dN"][there] if nxt else torch.zeros_like(stored), stored, s64[there, 2:3], s64[there, 3:4], nxt, w["w_next"])
    dr = torch.zeros(M, C, dtype=torch.float64)
    mag_r = torch.zeros_like(dr)
    dr[there], mag_r[there] = w["dR"][live] + dx, w["dR"][live].abs() + mag_x
    want, mag = w["dR"].clone(), torch.zeros(S, C, dtype=torch.float64)
    want[live], mag[live] = a * dr[there], a * mag_r[there]
    check("dR", dR, want, mag, dtype)
    assert torch.equal(dR.cpu()[rest], t["dR"][rest])
    du = beta * g * dr
    many = 64 + -(-M // 256) + 8 + 512 // 4
    if nxt:
        check("dw_next", got.dw_next, dw, mag_w, torch.float32, many)
        check("db_next", got.db_next, db, mag_b, torch.float32, many)
    dY, dw, db, mag_y, mag_w, mag_b = back64(du, w["Y"], s64[:, 0:1], s64[:, 1:2], post, w["w_post"])
    mag_du = abs(beta) * g.abs() * mag_r
    if post:  # du itself carries the errors of dr
        mag_y = back64(mag_du, w["Y"], s64[:, 0:1], s64[:, 1:2], post, w["w_post"])[3] * 2
    else:
        mag_y = mag_du
    dY[~there], mag_y[~there] = 0, 0
    check("dY", got.dY, dY, mag_y, dtype)
    if post:
        ym = (w["Y"].abs() + s64[:, 0:1].abs()) * s64[:, 1:2]
        check("dw_post", got.dw_post, dw, (mag_du * ym)[there].sum(0) * 2, torch.float32, many)
        if got.db_post is not None:
            check("db_post", got.db_post, db, mag_du[there].sum(0) * 2, torch.float32, many)
    if gate == "none":
        assert got.dgate is None
        return
    dg = beta * u * dr * (g * (1 - g) if gate == "sigmoid" else 1)
    mag = abs(beta) * mag_u * mag_r * 2
    dg[~there], mag[~there] = 0, 0
    if gate == "row":
        check("dgate", got.dgate, dg.sum(0), mag.sum(0), torch.float32, many)
    else:
        check("dgate", got.dgate, dg, mag, dtype)


@pytest.mark.gpu
def test_gradient_against_differences(lemo):
    """binary32, centred differences of a 64-bit sum of the results; step 2^-6: truncation and rounding stay below 1e-3 of the gradients' scale."""
    M, C, a, beta, eps = 3, 8, 0.7, 0.6, 1e-5
    t = inputs(torch.float32, M, M, C, 2, 2, "sigmoid", None, seed=5)
    d = {k: v.cuda() if v is not None else None for k, v in t.items()}
    how = dict(post=2, next=2, residual_scale=a, block_scale=beta, flags=lemo.GATE_SIGMOID)

    def loss(**change):
        x = {**d, **change}
        R = x["R"].clone()
        N, _ = lemo.lemo_norm_residual(x["Y"], R, None, gate=x["gate"], w_post=x["w_post"], b_post=x["b_post"], w_next=x["w_next"], b_next=x["b_next"],
                                       eps=eps, **how)
        return ((N.double() * d["dN"].double()).sum() + (R.double() * d["dR"].double()).sum()).item()

    R = d["R"].clone()
    _, stats = lemo.lemo_norm_residual(d["Y"], R, None, gate=d["gate"], w_post=d["w_post"], b_post=d["b_post"], w_next=d["w_next"], b_next=d["b_next"], eps=eps, **how)
    dR = d["dR"].clone()
    got = lemo.lemo_norm_residual_grad(d["dN"], dR, R, d["Y"], None, stats, gate=d["gate"], w_post=d["w_post"], b_post=d["b_post"], w_next=d["w_next"], **how)
    h = 2.0 ** -6
    for name, grad in (("R", dR), ("Y", got.dY), ("gate", got.dgate), ("w_post", got.dw_post), ("b_post", got.db_post), ("w_next", got.dw_next), ("b_next", got.db_next)):
        for at in (0, 5, d[name].numel() - 1):
            e = torch.zeros_like(d[name]).view(-1)
            e[at] = h
            e = e.view_as(d[name])
            slope = (loss(**{name: d[name] + e}) - loss(**{name: d[name] - e})) / (2 * h)
            assert abs(slope - grad.view(-1)[at].item()) <= 2e-3 * (1 + abs(slope)), (name, at, slope, grad.view(-1)[at].item())


@pytest.mark.gpu
def test_fused_and_separate_calls_give_the_same_bits(lemo):
    t = inputs(torch.bfloat16, 50, 80, 768, 1, 2, "rows", "kept", seed=9)
    d = {k: v.cuda() if v is not None else None for k, v in t.items()}
    how = dict(gate=d["gate"], post=1, w_post=d["w_post"], residual_scale=0.9, block_scale=0.5)
    R = d["R"].clone()
    N, stats = lemo.lemo_norm_residual(d["Y"], R, d["idx"], next=2, w_next=d["w_next"], b_next=d["b_next"], **how)
    S = d["R"].clone()
    lemo.lemo_norm_residual(d["Y"], S, d["idx"], next=0, **how)
    assert torch.equal(R, S)
    N1, stats1 = lemo.lemo_norm_residual(None, S, d["idx"], next=2, w_next=d["w_next"], b_next=d["b_next"])
    assert torch.equal(N, N1) and torch.equal(R, S) and torch.equal(stats[:, 2:], stats1[:, 2:]) and not stats1[:, :2].any()


@pytest.mark.gpu
def test_strides_results_in_the_place_of_operands_and_no_rows(lemo):
    M, S, C = 19, 40, 136
    t = inputs(torch.bfloat16, M, S, C, 1, 1, "rows", "kept", seed=3)
    d = {k: v.cuda() if v is not None else None for k, v in t.items()}

    def apart(x, extra):
        big = torch.full((x.shape[0], x.shape[1] + extra), 7.0, dtype=x.dtype, device="cuda")
        big[:, :x.shape[1]] = x
        return big[:, :x.shape[1]]

    how = dict(post=1, next=1, w_post=d["w_post"], w_next=d["w_next"])
    R = d["R"].clone()
    N, stats = lemo.lemo_norm_residual(d["Y"], R, d["idx"], gate=d["gate"], **how)
    R2, Y2 = apart(d["R"], 24), apart(d["Y"], 8)
    N2, stats2 = lemo.lemo_norm_residual(Y2, R2, d["idx"], gate=apart(d["gate"], 16), N=Y2, **how)
    assert torch.equal(R, R2) and torch.equal(N, N2) and torch.equal(stats, stats2) and N2.data_ptr() == Y2.data_ptr()
    assert (R2._base[:, C:] == 7).all() and (Y2._base[:, C:] == 7).all()
    dR, dR2 = d["dR"].clone(), apart(d["dR"], 40)
    got = lemo.lemo_norm_residual_grad(d["dN"], dR, R, d["Y"], d["idx"], stats, gate=d["gate"], **how)
    got2 = lemo.lemo_norm_residual_grad(apart(d["dN"], 8), dR2, R2, apart(d["Y"], 8), d["idx"], stats, gate=apart(d["gate"], 16), **how)
    assert torch.equal(dR, dR2) and all(torch.equal(x, y) for x, y in zip(got, got2) if x is not None)
    # no rows at all: nothing changes, the sums are zeros
    none = torch.empty(0, dtype=torch.int32, device="cuda")
    R3, empty = R.clone(), torch.empty(0, C, dtype=torch.bfloat16, device="cuda")
    N3, stats3 = lemo.lemo_norm_residual(empty, R3, none, **how)
    got3 = lemo.lemo_norm_residual_grad(empty, dR2, R3, empty, none, stats3, **how)
    assert torch.equal(R3, R) and N3.shape == (0, C) and torch.equal(dR, dR2)
    assert not got3.dw_next.any() and not got3.dw_post.any() and got3.dY.shape == (0, C)


@pytest.mark.gpu
def test_replayed_graphs_and_other_streams(lemo):
    M, S, C = 300, 500, 1024
    t = inputs(torch.bfloat16, M, S, C, 1, 1, "row", "kept", seed=4)
    d = {k: v.cuda() if v is not None else None for k, v in t.items()}
    how = dict(gate=d["gate"], post=1, next=1, w_post=d["w_post"], w_next=d["w_next"], residual_scale=0.5, block_scale=0.5)
    R, dR = d["R"].clone(), d["dR"].clone()

    def both():
        N, stats = lemo.lemo_norm_residual(d["Y"], R, d["idx"], **how)
        return (N, stats, *lemo.lemo_norm_residual_grad(d["dN"], dR, R, d["Y"], d["idx"], stats, **how))

    def again():
        R.copy_(d["R"])
        dR.copy_(d["dR"])

    want = [x.clone() for x in both() if x is not None] + [R.clone(), dR.clone()]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        again()
        got = [x for x in both() if x is not None] + [R, dR]
    torch.cuda.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(want, got))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = [x for x in both() if x is not None]
    for _ in range(3):
        again()
        for x in out:
            x.fill_(3.0)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(want, out + [R, dR]))


def test_argument_errors():
    """Refused on the host, before any launch: the addresses are never touched."""
    from paper_2501_09767_amd import lemo
    lib = lemo._lib
    P = [0x10000 * (i + 1) for i in range(20)]
    names = "Y ldy gate ldg R ldr S idx M wp bp post wn bn next eps a beta N ldn stats C dt flags stream".split()
    ok = dict(Y=P[0], ldy=64, gate=P[1], ldg=64, R=P[2], ldr=64, S=100, idx=P[3], M=10, wp=P[4], bp=P[5], post=1, wn=P[6], bn=P[7], next=2, eps=1e-5, a=1.0,
              beta=1.0, N=P[8], ldn=64, stats=P[9], C=64, dt=1, flags=0, stream=None)
    f = lambda **kw: lib.lemo_norm_residual(*[dict(ok, **kw)[k] for k in names])  # noqa: E731
    assert f(dt=3) == -3 and f(R=None) == -1 and f(N=None) == -1
    assert f(post=3) == -2 and f(next=-1) == -2 and f(flags=2) == -2 and f(eps=-1.0) == -2 and f(eps=math.nan) == -2 and f(a=math.inf) == -2 and f(beta=math.nan) == -2
    assert f(Y=None) == -2 and f(Y=None, gate=None) == -2 and f(Y=None, gate=None, post=0, next=0) == -2 and f(gate=None, flags=1) == -2
    assert f(S=0) == -2 and f(M=-1) == -2 and f(M=101) == -2 and f(C=0) == -2 and f(ldy=56) == -2 and f(ldg=8) == -2 and f(ldr=32) == -2 and f(ldn=63) == -2
    assert f(C=60) == -6 and f(C=16392, ldy=16392, ldg=0, ldr=16392, ldn=16392) == -6 and f(dt=0, C=62) == -6
    assert f(Y=P[0] + 8) == -5 and f(ldr=68) == -5 and f(wn=P[6] + 4) == -5 and f(stats=P[9] + 4) == -5 and f(idx=P[3] + 2) == -5 and f(gate=P[1] + 2, ldg=0) == -5
    assert f(M=0) == 0
    n = ctypes.c_size_t()
    assert lib.lemo_norm_residual_grad_workspace_bytes(10, 64, ctypes.byref(n)) == 0 and n.value == 10 * 5 * 64 * 4
    assert lib.lemo_norm_residual_grad_workspace_bytes(-1, 64, ctypes.byref(n)) == -2 and lib.lemo_norm_residual_grad_workspace_bytes(1, 64, None) == -1
    names = ("dN lddn dR lddr S R ldr Y ldy gate ldg idx M wp bp post wn next a beta stats dY lddy dgate lddg dwp dbp dwn dbn dgs C dt flags ws wsb "
             "stream").split()
    ok = dict(dN=P[0], lddn=64, dR=P[1], lddr=64, S=100, R=P[2], ldr=64, Y=P[3], ldy=64, gate=P[4], ldg=64, idx=P[5], M=10, wp=P[6], bp=P[7], post=1, wn=P[8],
              next=2, a=1.0, beta=1.0, stats=P[9], dY=P[10], lddy=64, dgate=P[11], lddg=64, dwp=P[12], dbp=P[13], dwn=P[14], dbn=P[15], dgs=None, C=64, dt=1,
              flags=0, ws=P[16], wsb=10 * 5 * 64 * 4, stream=None)
    f = lambda **kw: lib.lemo_norm_residual_grad(*[dict(ok, **kw)[k] for k in names])  # noqa: E731
    assert f(dt=2) == -3 and f(dR=None) == -1 and f(dN=None) == -1 and f(R=None) == -1 and f(stats=None) == -1 and f(ws=None) == -1
    assert f(Y=None) == -2 and f(next=0) == -2 and f(post=0) == -2 and f(gate=None) == -2 and f(ldg=0) == -2 and f(M=101) == -2 and f(lddy=32) == -2 and f(beta=math.inf) == -2
    assert f(gate=None, dgate=None, flags=1) == -2 and f(post=5) == -2 and f(flags=4) == -2
    assert f(wsb=100) == -4 and f(ws=P[16] + 16) == -5 and f(dwp=P[12] + 2) == -5 and f(lddr=66) == -5 and f(C=60) == -6


def test_binding_refuses_tensors_that_do_not_fit(lemo):
    with pytest.raises(ValueError):
        lemo.lemo_norm_residual(torch.zeros(2, 8), torch.zeros(2, 8))  # not on the GPU

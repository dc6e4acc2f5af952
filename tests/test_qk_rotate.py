"""Norms and rotation of queries and keys, their gradients and their form for single tokens, against the formulas in 64 bits.

Tolerances: a stored value is off by at most half a step of its type and by the binary32 arithmetic before it: every term that enters a
result passes through fewer than 64 roundings of 2^-24 (the norm's sums, products, and cos and sin, which are within 8 * 2^-24 of 1 from the
64-bit angle's), so 64 * 2^-24 of the terms' magnitudes bounds it.  Sums over the tokens: a lane adds at most 4 * (M / 256 + 1) terms, then up
to 64 places, rows / 32 parts and 32 threads are added: 256 more for the sizes here."""
import ctypes
import math

import pytest
import torch

U = 2.0 ** -24


@pytest.fixture(scope="module")
def lemo():
    from paper_2501_09767_amd import lemo
    return lemo


def spin(x, angle, pairs, amplitude, back=False):
    """Rotates the first channels of x [M,heads,d] by angle [M,rot/2] (64 bits); with absolute values in, the magnitudes of the terms."""
    rot, size = 2 * angle.shape[1], back is None
    cos, sin = torch.cos(angle)[:, None] * amplitude, torch.sin(angle)[:, None] * amplitude
    if size:
        cos, sin = cos.abs().clamp(min=abs(amplitude) / 8), sin.abs().clamp(min=abs(amplitude) / 8)  # (errors of cos and sin are absolute)
    elif back:
        sin = -sin
    i = torch.arange(rot // 2)
    a, b = (2 * i, 2 * i + 1) if pairs else (i, i + rot // 2)
    y = x.clone()
    y[:, :, a] = x[:, :, a] * cos + (1 if size else -1) * x[:, :, b] * sin
    y[:, :, b] = x[:, :, b] * cos + x[:, :, a] * sin
    return y


def norm64(x, mode, eps):
    """xhat, 1 / deviation, magnitude of xhat's terms."""
    if mode == 0:
        return x, torch.ones(*x.shape[:2], 1, dtype=torch.float64), x.abs()
    mean = x.mean(2, keepdim=True) if mode == 2 else torch.zeros(*x.shape[:2], 1, dtype=torch.float64)
    rstd = ((x - mean).square().mean(2, keepdim=True) + eps).rsqrt()
    return (x - mean) * rstd, rstd, (x.abs() + (x.abs().mean(2, keepdim=True) if mode == 2 else 0)) * rstd


def forward64(x, w, mode, eps, angle, pairs, amplitude):
    xh, _, mag = norm64(x, mode, eps)
    w = 1.0 if w is None else w
    return spin(xh * w, angle, pairs, amplitude), spin(mag * (w.abs() if torch.is_tensor(w) else 1.0), angle, pairs, amplitude, None)


def back64(dy, x, w, mode, eps, angle, pairs, amplitude, per_head):
    t, mag_t = spin(dy, angle, pairs, amplitude, True), spin(dy.abs(), angle, pairs, amplitude, None)
    if mode == 0:
        return t, None, mag_t, None
    xh, rstd, xm = norm64(x, mode, eps)
    over = 0 if per_head else (0, 1)
    dw, mag_w = (t * xh).sum(over), (mag_t * xm).sum(over)
    w = torch.ones(x.shape[2], dtype=torch.float64) if w is None else w
    t, mag_t = t * w, mag_t * w.abs()
    dx = rstd * (t - xh * (t * xh).mean(2, keepdim=True) - (t.mean(2, keepdim=True) if mode == 2 else 0))
    return dx, dw, rstd * (mag_t + xm * (mag_t * xm).mean(2, keepdim=True) + mag_t.mean(2, keepdim=True)), mag_w


def check(name, got, want, mag, dtype, roundings=64):
    half = torch.finfo(dtype).eps / 2
    got = got.double().cpu()
    assert got.shape == want.shape and torch.isfinite(got).all(), name
    off = (got - want).abs() - (half * want.abs() + roundings * U * (1 + half) * mag)
    assert off.numel() == 0 or off.max() <= 1e-38, f"{name}: {off.max().item():.3g} over the bound"


SHAPES = [  # dtype, M, H, H_kv, d, rot, norm, weights ("shared", "heads", None), pairs, positions, pos_start, amplitude
    (torch.bfloat16, 1, 1, 1, 64, 64, 1, "shared", False, None, 0, 1.0),
    (torch.bfloat16, 5, 32, 8, 128, 128, 1, "shared", False, None, 7, 1.0),
    (torch.bfloat16, 77, 12, 12, 64, 32, 2, "heads", True, "far", 0, 1.2),
    (torch.bfloat16, 300, 33, 11, 128, 64, 1, "heads", False, "kept", 0, 1.0),
    (torch.bfloat16, 2050, 4, 2, 64, 64, 2, "shared", True, None, -100, 0.5),
    (torch.bfloat16, 2600, 16, 16, 128, 128, 0, None, False, "kept", 0, 1.0),
    (torch.bfloat16, 64, 40, 40, 64, 0, 1, "shared", False, None, 0, 1.0),
    (torch.bfloat16, 9, 7, 0, 128, 96, 2, None, False, "far", 0, 1.0),
    (torch.bfloat16, 13, 0, 3, 64, 16, 1, "shared", True, "far", 2 ** 30, 1.0),
    (torch.float32, 1, 3, 1, 128, 128, 2, "shared", True, "far", 0, 1.0),
    (torch.float32, 999, 12, 12, 64, 64, 1, "shared", False, None, 0, 1.0),
    (torch.float32, 130, 20, 5, 128, 40, 1, "heads", False, "kept", 3, 1.0),
    (torch.float32, 4100, 2, 1, 64, 32, 1, "heads", True, None, 0, 0.9),
    (torch.float32, 31, 70, 10, 64, 8, 0, None, True, "far", 0, 1.0),
]


def inputs(dtype, M, H, Hkv, d, rot, norm, weights, pairs, where, start, amplitude, seed):
    g = torch.Generator().manual_seed(seed)
    n = lambda *s, std=1.0: (torch.randn(*s, generator=g) * std).to(dtype)  # noqa: E731
    t = dict(Q=n(M, H, d, std=1.5) + 0.25, K=n(M, Hkv, d) - 0.5, dQ=n(M, H, d, std=0.3), dK=n(M, Hkv, d, std=0.3))
    for name, heads in (("w_q", H), ("w_k", Hkv)):
        t[name] = None if weights is None or heads == 0 else (1 + n(*((heads, d) if weights == "heads" else (d,)), std=0.3)).to(dtype)
    t["inv_freq"] = (10000.0 ** (-torch.arange(0, rot, 2).double() / max(rot, 1))).float() if rot else None
    t["positions"] = None if where is None else torch.randint(-5, 40 * M, (M,), generator=g).int() if where == "kept" else \
        torch.randint(-2 ** 31, 2 ** 31, (M,), generator=g).int() if start == 0 else torch.randint(0, 2 ** 30, (M,), generator=g).int()
    place = (torch.arange(M) if t["positions"] is None else t["positions"].long()) + start
    angle = place.double()[:, None] * (t["inv_freq"].double()[None] if rot else torch.zeros(1, 0, dtype=torch.float64))
    return t, angle


def on_gpu(t):
    return {k: None if v is None else v.cuda() for k, v in t.items()}


@pytest.mark.gpu
@pytest.mark.parametrize("case", range(len(SHAPES)))
def test_forward_and_gradient_against_64_bits(lemo, case):
    dtype, M, H, Hkv, d, rot, norm, weights, pairs, where, start, amplitude = SHAPES[case]
    print(SHAPES[case], flush=True)
    t, angle = inputs(*SHAPES[case], seed=case)
    c = on_gpu(t)
    sides = [(n, x) for n, x in (("Q", H), ("K", Hkv)) if x]
    eps = 1e-5
    how = dict(pos_start=start, norm=norm, w_q=c["w_q"], w_k=c["w_k"], eps=eps, amplitude=amplitude, flags=lemo.ROTATE_PAIRS if pairs else 0)
    Q, K = c["Q"] if H else None, c["K"] if Hkv else None
    out = dict(zip("QK", lemo.lemo_qk_rotate(Q, K, c["inv_freq"], c["positions"], **how)))
    dQ, dK = c["dQ"] if H else None, c["dK"] if Hkv else None
    got = lemo.lemo_qk_rotate_grad(dQ, dK, Q, K, c["inv_freq"], c["positions"], **how)
    for n, _ in sides:
        w = t["w_" + n.lower()]
        w = None if w is None else w.double()
        want, mag = forward64(t[n].double(), w, norm, eps, angle, pairs, amplitude)
        check(n, out[n], want, mag, dtype)
        dx, dw, mag_x, mag_w = back64(t["d" + n].double(), t[n].double(), w, norm, eps, angle, pairs, amplitude, weights == "heads")
        check("d" + n, getattr(got, "d" + n), dx, mag_x, dtype)
        if w is not None:
            check("dw of " + n, getattr(got, "dw_" + n.lower()), dw, mag_w, torch.float32, 320)
    assert (out["Q"] is None) == (H == 0) and (got.dK is None) == (Hkv == 0)
    assert all((got[2 + i] is None) == (c[n] is None) for i, n in enumerate(("w_q", "w_k")))


@pytest.mark.gpu
def test_gradient_against_differences(lemo):
    """binary32, centred differences of a 64-bit sum of the results; step 2^-6: truncation (h^2 / 6 of third derivatives of the order of 1) and rounding
    (2^-24 * 128 terms / h) stay below 1e-3 of the gradients' scale."""
    shape = (torch.float32, 3, 2, 1, 64, 32, 2, "heads", False, "kept", 0, 1.1)
    t, _ = inputs(*shape, seed=11)
    c = on_gpu(t)

    def total(**change):
        x = {**c, **change}
        Q, K = lemo.lemo_qk_rotate(x["Q"], x["K"], c["inv_freq"], c["positions"], norm=2, w_q=x["w_q"], w_k=x["w_k"], amplitude=1.1)
        return ((Q.double() * c["dQ"].double()).sum() + (K.double() * c["dK"].double()).sum()).item()

    got = lemo.lemo_qk_rotate_grad(c["dQ"], c["dK"], c["Q"], c["K"], c["inv_freq"], c["positions"], norm=2, w_q=c["w_q"], w_k=c["w_k"], amplitude=1.1)
    h = 2.0 ** -6
    for name, grad in (("Q", got.dQ), ("K", got.dK), ("w_q", got.dw_q), ("w_k", got.dw_k)):
        for at in (0, 17, 40, grad.numel() - 1):
            e = torch.zeros(grad.numel(), device="cuda")
            e[at] = h
            e = e.view_as(c[name])
            slope = (total(**{name: c[name] + e}) - total(**{name: c[name] - e})) / (2 * h)
            assert abs(slope - grad.reshape(-1)[at].item()) <= 2e-3 * (1 + abs(slope)), (name, at, slope, grad.reshape(-1)[at].item())


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_slices_of_a_fused_projection_other_layouts_and_results_in_place(lemo, dtype):
    M, H, Hkv, d = 41, 6, 2, 128
    g = torch.Generator().manual_seed(2)
    qkv = torch.randn(M, H + 2 * Hkv, d, generator=g).to(dtype).cuda()
    w = (1 + torch.randn(d, generator=g) / 4).to(dtype).cuda()
    f = (10000.0 ** (-torch.arange(0, d, 2) / d)).float().cuda()
    Q, K = qkv[:, :H], qkv[:, H:H + Hkv]
    how = dict(w_q=w, w_k=w)
    want = lemo.lemo_qk_rotate(Q.contiguous(), K.contiguous(), f, **how)
    got = lemo.lemo_qk_rotate(Q, K, f, **how)
    assert all(torch.equal(x, y) for x, y in zip(want, got))
    by_head = [torch.empty(n, M, d, dtype=dtype, device="cuda").transpose(0, 1) for n in (H, Hkv)]
    lemo.lemo_qk_rotate(Q, K, f, Q_out=by_head[0], K_out=by_head[1], **how)
    assert all(torch.equal(x, y) for x, y in zip(want, by_head))
    dQ, dK = torch.randn(M, H, d, generator=g).to(dtype).cuda(), torch.randn(M, Hkv, d, generator=g).to(dtype).cuda()
    back = lemo.lemo_qk_rotate_grad(dQ, dK, Q, K, f, **how)
    same = lemo.lemo_qk_rotate_grad(dQ, dK, Q.contiguous(), K.contiguous(), f, dQ=dQ, dK=dK, **how)
    assert same.dQ is dQ and all(torch.equal(x, y) for x, y in zip(back, same))
    values = qkv[:, H + Hkv:].clone()
    lemo.lemo_qk_rotate(Q, K, f, Q_out=Q, K_out=K, **how)
    assert torch.equal(Q, want[0]) and torch.equal(K, want[1]) and torch.equal(qkv[:, H + Hkv:], values)
    # one token more or less changes no other: rows do not depend on how many there are
    few = lemo.lemo_qk_rotate(by_head[0][:7].contiguous(), None, f, w_q=w)[0]
    many = lemo.lemo_qk_rotate(by_head[0].contiguous(), None, f, w_q=w)[0]
    assert torch.equal(few, many[:7])


@pytest.mark.gpu
def test_values_that_are_not_finite_stay_in_their_head(lemo):
    M, H, d = 6, 8, 64
    g = torch.Generator().manual_seed(3)
    Q = torch.randn(M, H, d, generator=g).bfloat16().cuda()
    f = (10000.0 ** (-torch.arange(0, d, 2) / d)).float().cuda()
    want, _ = lemo.lemo_qk_rotate(Q, None, f)
    back = lemo.lemo_qk_rotate_grad(Q, None, Q, None, f).dQ
    bad = Q.clone()
    bad[2, 3, 5], bad[4, 0, 63] = math.inf, math.nan
    got, _ = lemo.lemo_qk_rotate(bad, None, f)
    other = torch.ones(M, H, dtype=torch.bool)
    other[2, 3] = other[4, 0] = False
    other = other.cuda()
    assert torch.equal(got[other], want[other]) and not torch.isfinite(got[2, 3]).all() and torch.isnan(got[4, 0]).all()
    assert torch.equal(lemo.lemo_qk_rotate_grad(Q, None, bad, None, f).dQ[other], back[other])
    # a head of zeros: eps keeps it finite
    zero = torch.zeros_like(Q)
    assert not lemo.lemo_qk_rotate(zero, None, f)[0].any()


@pytest.mark.gpu
def test_no_tokens(lemo):
    d = 64
    f = torch.ones(d // 2, device="cuda")
    none, w = torch.empty(0, 4, d, dtype=torch.bfloat16, device="cuda"), torch.ones(d, dtype=torch.bfloat16, device="cuda")
    Q, K = lemo.lemo_qk_rotate(none, none, f, w_q=w, w_k=w)
    assert Q.shape == K.shape == (0, 4, d)
    got = lemo.lemo_qk_rotate_grad(none, none, none, none, f, w_q=w, w_k=w)
    assert got.dQ.shape == (0, 4, d) and not got.dw_q.any() and not got.dw_k.any()
    per_head = lemo.lemo_qk_rotate_grad(none, None, none, None, f, w_q=w.expand(4, d).contiguous())
    assert per_head.dw_q.shape == (4, d) and not per_head.dw_q.any()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype, B, S, H, Hkv, d, norm", [(torch.bfloat16, 1, 5, 32, 8, 128, 1), (torch.bfloat16, 9, 33, 12, 12, 64, 2), (torch.float32, 70, 7, 4, 1, 128, 1),
                                                          (torch.bfloat16, 2500, 3, 2, 1, 64, 0)])
def test_single_tokens_are_the_rows_of_a_prompt(lemo, dtype, B, S, H, Hkv, d, norm):
    g = torch.Generator().manual_seed(B)
    qkv = torch.randn(B, H + 2 * Hkv, d, generator=g).to(dtype).cuda()
    Q, K, V = qkv[:, :H], qkv[:, H:H + Hkv], qkv[:, H + Hkv:]
    f = (10000.0 ** (-torch.arange(0, d, 2) / d)).float().cuda()
    w = (1 + torch.randn(d, generator=g) / 4).to(dtype).cuda() if norm else None
    lengths = torch.randint(1, S + 1, (B,), generator=g).int()
    odd = min(3, B - 1)
    lengths[:odd] = torch.tensor([0, -4, S + 5])[:odd].int()
    lengths = lengths.cuda()
    taken = lengths.clamp(0, S)
    caches = [torch.randn(B, Hkv, S, d, generator=g).to(dtype).cuda().transpose(1, 2) for _ in range(2)]  # heads before tokens
    want = [c.clone() for c in caches]
    rows = lemo.lemo_qk_rotate(Q, K, f, (taken - 1).int(), norm=norm, w_q=w, w_k=w)
    live = (taken > 0).nonzero().squeeze(1)
    want[0][live, taken[live].long() - 1] = rows[1][live]
    want[1][live, taken[live].long() - 1] = V[live]
    got = lemo.lemo_qk_rotate_step(Q, K, V, caches[0], caches[1], lengths, f, norm=norm, w_q=w, w_k=w)
    assert all(torch.equal(x, y) for x, y in zip(caches, want))
    assert torch.equal(got[live], rows[0][live]) and not got[taken == 0].any()
    # keys alone
    keys = want[0].clone()
    keys[live, taken[live].long() - 1] = 0
    lemo.lemo_qk_rotate_step(Q, K, None, keys, None, lengths, f, norm=norm, w_q=w, w_k=w)
    assert torch.equal(keys, want[0])


@pytest.mark.gpu
def test_replayed_graphs_and_other_streams(lemo):
    shape = (torch.bfloat16, 2100, 8, 4, 128, 128, 1, "shared", False, "kept", 0, 1.0)
    t, _ = inputs(*shape, seed=21)
    c = on_gpu(t)
    lengths = torch.tensor([3], dtype=torch.int32, device="cuda")
    cache = torch.zeros(1, 8, 4, 128, dtype=torch.bfloat16, device="cuda")

    def all_three():
        out = lemo.lemo_qk_rotate(c["Q"], c["K"], c["inv_freq"], c["positions"], w_q=c["w_q"], w_k=c["w_k"])
        back = lemo.lemo_qk_rotate_grad(c["dQ"], c["dK"], c["Q"], c["K"], c["inv_freq"], c["positions"], w_q=c["w_q"], w_k=c["w_k"])
        return [*out, *back, lemo.lemo_qk_rotate_step(c["Q"][:1], c["K"][:1], None, cache, None, lengths, c["inv_freq"], w_q=c["w_q"], w_k=c["w_k"])]

    want = [x.clone() for x in all_three()] + [cache.clone()]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        cache.zero_()
        got = all_three() + [cache]
    torch.cuda.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(want, got))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = all_three()
    for n in (3, 5, 8):  # the length is read at each replay
        lengths.fill_(n)
        cache.zero_()
        for x in out:
            x.fill_(3.0)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(want[:6], out[:6]))
        assert cache[0, n - 1].any() and not cache[0, [i for i in range(8) if i != n - 1]].any()


def test_argument_errors():
    """Refused on the host, before any launch: the addresses are never touched."""
    from paper_2501_09767_amd import lemo
    lib = lemo._lib
    P = [0x10000 * (i + 1) for i in range(20)]
    names = "Q qt qh K kt kh M H Hkv d dt pos start f rot amp norm wq wk eps flags Qo qot qoh Ko kot koh stream".split()
    ok = dict(Q=P[0], qt=512, qh=128, K=P[1], kt=256, kh=128, M=10, H=4, Hkv=2, d=128, dt=1, pos=P[2], start=0, f=P[3], rot=128, amp=1.0, norm=1, wq=P[4], wk=P[5],
              eps=1e-6, flags=0, Qo=P[6], qot=512, qoh=128, Ko=P[7], kot=256, koh=128, stream=None)
    f = lambda **kw: lib.lemo_qk_rotate(*[dict(ok, **kw)[k] for k in names])  # noqa: E731
    assert f(dt=2) == -3 and f(Q=None) == -1 and f(Ko=None) == -1 and f(f=None) == -1
    assert f(norm=3) == -2 and f(flags=4) == -2 and f(M=-1) == -2 and f(M=2 ** 31) == -2 and f(H=-1) == -2 and f(H=0, Hkv=0) == -2 and f(rot=130) == -2 and f(rot=-16) == -2
    assert f(eps=-1.0) == -2 and f(eps=math.nan) == -2 and f(amp=math.inf) == -2 and f(start=2 ** 31) == -2 and f(start=-2 ** 31) == -2
    assert f(qt=-8) == -2 and f(qot=0) == -2 and f(koh=64) == -2
    assert f(d=96, rot=96) == -6 and f(rot=120) == -6 and f(dt=0, rot=124) == -6 and f(H=65535) == -6
    assert f(Q=P[0] + 8) == -5 and f(qh=132) == -5 and f(pos=P[2] + 2) == -5 and f(f=P[3] + 2) == -5 and f(wq=P[4] + 4) == -5
    assert f(M=0) == 0
    n = ctypes.c_size_t()
    need = lib.lemo_qk_rotate_grad_workspace_bytes
    assert need(10, 4, 2, 128, 1, 0, ctypes.byref(n)) == 0 and n.value > 0 and need(10, 4, 2, 128, 1, 0, None) == -1
    assert need(-1, 4, 2, 128, 1, 0, ctypes.byref(n)) == -2 and need(1, 4, 2, 96, 1, 0, ctypes.byref(n)) == -6
    assert need(2 ** 31 - 1, 65000, 535, 128, 1, 2, ctypes.byref(n)) == 0
    names = "dQo a b dKo c e Q qt qh K kt kh M H Hkv d dt pos start f rot amp norm wq wk eps flags dQ g h dK i j dwq dwk ws wsb stream".split()
    ok = dict(ok, dQo=P[6], a=512, b=128, dKo=P[7], c=256, e=128, dQ=P[8], g=512, h=128, dK=P[9], i=256, j=128, dwq=P[10], dwk=P[11], ws=P[12], wsb=1 << 20)
    f = lambda **kw: lib.lemo_qk_rotate_grad(*[dict(ok, **kw)[k] for k in names])  # noqa: E731
    assert f(dt=5) == -3 and f(dQo=None) == -1 and f(Q=None) == -1 and f(dK=None) == -1 and f(ws=None) == -1
    assert f(norm=0) == -2 and f(H=0) == -2 and f(g=8) == -2 and f(wsb=16) == -4 and f(ws=P[12] + 16) == -5 and f(dwq=P[10] + 2) == -5 and f(a=516) == -5
    assert f(M=0, dwq=None, dwk=None) == 0
    names = ("Q qt qh K kt kh V vt vh B S H Hkv d dt len f rot amp norm wq wk eps flags Qo qot qoh Kc ks kct kch Vc vs vct vch stream").split()
    ok = dict(ok, V=P[13], vt=256, vh=128, B=3, S=100, len=P[14], Kc=P[15], ks=25600, kct=256, kch=128, Vc=P[16], vs=25600, vct=256, vch=128)
    f = lambda **kw: lib.lemo_qk_rotate_step(*[dict(ok, **kw)[k] for k in names])  # noqa: E731
    assert f(V=None) == -2 and f(Vc=None) == -2 and f(S=0) == -2 and f(S=2 ** 31) == -2 and f(len=None) == -1 and f(Kc=None) == -1
    assert f(ks=25604) == -5 and f(len=P[14] + 2) == -5 and f(kct=64) == -2 and f(ks=0) == -2 and f(vs=-8) == -2 and f(B=-1) == -2
    assert f(B=0) == 0


def test_results_whose_rows_lie_on_each_other_are_refused():
    """Refused on the host, in whatever order the dimensions lie; what is not refused for its strides is for the positions' or lengths' address, looked at after them."""
    from paper_2501_09767_amd import lemo
    lib = lemo._lib
    A = 0x10000

    def rotate(M, H, ts, hs):  # (heads of queries only)
        return lib.lemo_qk_rotate(A, 4096, 128, None, 0, 0, M, H, 0, 128, 1, A + 2, 0, A, 128, 1.0, 1, None, None, 1e-6, 0, A, ts, hs, None, 0, 0, None)

    def step(B, S, H, seq, tok, head):  # (heads of keys only)
        return lib.lemo_qk_rotate_step(None, 0, 0, A, 4096, 128, None, 0, 0, B, S, 0, H, 128, 1, A + 2, A, 128, 1.0, 1, None, None, 1e-6, 0, None, 0, 0, A, seq, tok, head,
                                       None, 0, 0, 0, None)
    assert rotate(10, 4, 512, 128) == -5 and rotate(10, 4, 128, 1280) == -5 and rotate(1, 4, 0, 128) == -5 and rotate(10, 1, 128, 0) == -5
    for ts, hs in ((128, 128), (384, 128), (128, 1152), (512, 0), (0, 1280), (504, 128)):
        assert rotate(10, 4, ts, hs) == -2, (ts, hs)
    assert step(3, 100, 2, 25600, 256, 128) == -5 and step(3, 100, 2, 256, 768, 128) == -5 and step(3, 100, 2, 25600, 128, 12800) == -5 and step(1, 100, 2, 0, 256, 128) == -5
    for seq, tok, head in ((256, 256, 128), (25472, 256, 128), (128, 256, 128), (256, 512, 128), (25600, 256, 0), (2 ** 62, 2 ** 62, 128)):
        assert step(3, 100, 2, seq, tok, head) == -2, (seq, tok, head)


def test_binding_refuses_tensors_that_do_not_fit(lemo):
    with pytest.raises(ValueError):
        lemo.lemo_qk_rotate(torch.zeros(2, 1, 64), None, None)  # not on the GPU
    with pytest.raises(ValueError):
        lemo.lemo_qk_rotate(None, None, None)

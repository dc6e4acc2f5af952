"""What a fine-tuning step has before the scoring and behind a block: norms and rotation of queries and keys, dropout into the
residual rows, and the loss over the vocabulary; in plain torch (32 bits, rounded once at the end), and as the calls of the public
binding that compute the same.

Seven kinds of pass:

  rotate       norm of every head of the queries and keys, and the rotation by their tokens' positions
  rotate_grad  gradients of that: queries, keys, norm weights
  rotate_step  the same for one new token of each sequence of a batch, keys and values written to their caches
  drop         dropout of a block's result and its add into the residual rows, the mask from a counter-based generator
  drop_grad    its gradient, the mask formed again
  loss         cross entropy over a vocabulary from hidden rows and the head's weight
  loss_grad    its gradients: hidden rows and weight

Sizes are those of this repository's own configurations (workloads.CONFIGS), its tests' ragged lengths, and generic layer widths and
vocabularies; `draw` spreads over the ranges in between.
"""
import math

import torch

own = False


def listed():
    return [
        # one sequence answered token by token over a long cache: latency decides
        _step("rotate_step_1", B=1, S=32768, H=32, H_kv=8, d=128),
        # a batch of conversations of different lengths
        _step("rotate_step_64", B=64, S=8192, H=32, H_kv=32, d=128),
        # every token of the long-context layer with grouped queries
        _rotate("rotate_32k_gqa", "rotate", M=32768, H=32, H_kv=8, d=128, rot=128, norm="rms"),
        # gradients of the usual fine-tuning sample, every head with its own keys
        _rotate("rotate_grad_8k", "rotate_grad", M=8192, H=32, H_kv=32, d=128, rot=128, norm="rms"),
        # gradients at the kept tokens of a small fp32 model: centred norms with weights for each head, half of a head turned, adjacent pairs
        _rotate("rotate_grad_999_fp32", "rotate_grad", M=999, H=12, H_kv=12, d=64, rot=32, norm="layer", per_head=True, pairs=True, kept=True, dtype="f32"),
        # the rows of a few tokens
        _drop("drop_8_rows", "drop", S=8, M=8, C=4096, p=0.1),
        # the kept rows of the 32K-token layer
        _drop("drop_32k_kept", "drop", S=32768, M=9856, C=4096, p=0.1),
        # gradient of a small fp32 model's sample of odd length
        _drop("drop_grad_2999_fp32", "drop_grad", S=2999, M=2999, C=768, p=0.25, dtype="f32"),
        # how likely a few tokens are, as a server of a small vocabulary is asked
        _loss("loss_16_rows", "loss", S=16, M=16, C=4096, V=32000),
        # the kept tokens of a fine-tuning sample, a large vocabulary
        _loss("loss_8k", "loss", S=16384, M=8192, C=4096, V=131072),
        # gradients of a small fp32 model over an odd vocabulary, its logits capped, its labels smoothed
        _loss("loss_grad_777_fp32", "loss_grad", S=1024, M=777, C=768, V=50001, softcap=30.0, smoothing=0.1, z_weight=1e-4, weights="rows", dtype="f32"),
        # gradients of that fine-tuning sample
        _loss("loss_grad_4k", "loss_grad", S=4096, M=4096, C=4096, V=131072, z_weight=1e-4),
    ]


def _rotate(name, kind, *, M, H, H_kv, d, rot, norm, per_head=False, pairs=False, kept=False, dtype="bf16"):
    return {"name": name, "kind": kind, "M": M, "H": H, "H_kv": H_kv, "d": d, "rot": rot, "norm": norm, "per_head": per_head, "pairs": pairs,
            "kept": kept, "dtype": dtype}


def _step(name, *, B, S, H, H_kv, d):
    return {"name": name, "kind": "rotate_step", "B": B, "S": S, "H": H, "H_kv": H_kv, "d": d, "rot": d, "norm": "rms", "per_head": False, "pairs": False,
            "dtype": "bf16"}


def _drop(name, kind, *, S, M, C, p, dtype="bf16"):
    return {"name": name, "kind": kind, "S": S, "M": M, "C": C, "p": p, "dtype": dtype}


def _loss(name, kind, *, S, M, C, V, softcap=0.0, smoothing=0.0, z_weight=0.0, weights="mean", dtype="bf16"):
    return {"name": name, "kind": kind, "S": S, "M": M, "C": C, "V": V, "softcap": softcap, "smoothing": smoothing, "z_weight": z_weight,
            "weights": weights, "dtype": dtype}


# (query heads, key heads, head size) of the layers a case is drawn for
_HEADS = [(4, 4, 64), (12, 12, 64), (16, 4, 64), (16, 16, 128), (32, 8, 128), (32, 32, 128)]
_WIDTHS = [256, 768, 1024, 2048, 4096]


def _spread(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["rotate", "rotate_grad", "rotate_step", "drop", "drop_grad", "loss", "loss", "loss_grad", "loss_grad"])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    if kind == "rotate_step":
        H, H_kv, d = rng.choice(_HEADS)
        B = _spread(rng, 1, 64)
        case = _step("", B=B, S=min(_spread(rng, 500, 32768), (1 << 19) // B), H=H, H_kv=H_kv, d=d)
    elif kind in ("rotate", "rotate_grad"):
        H, H_kv, d = rng.choice(_HEADS)
        case = _rotate("", kind, M=_spread(rng, 1, 32768 if kind == "rotate" else 8192), H=H, H_kv=H_kv, d=d, rot=rng.choice([d, d, d // 2]),
                       norm=rng.choice(["rms", "rms", "layer", "none"]), per_head=rng.random() < 0.3, pairs=rng.random() < 0.3, kept=rng.random() < 0.5,
                       dtype=dtype)
    elif kind in ("drop", "drop_grad"):
        C = rng.choice(_WIDTHS)
        S = min(_spread(rng, 1, 32768), (1 << 25) // C)
        case = _drop("", kind, S=S, M=max(1, int(S * rng.choice([1.0, 0.5, 0.3]))), C=C, p=rng.choice([0.02, 0.05, 0.1, 0.25, 0.5]), dtype=dtype)
    else:
        C, V = rng.choice(_WIDTHS), _spread(rng, 1000, 131072)
        # fp32 products are ten times as slow
        most = (1 << (41 if dtype == "bf16" else 37)) // (C * V)
        S = max(1, min(_spread(rng, 1, 8192), most))
        case = _loss("", kind, S=S, M=max(1, int(S * rng.choice([1.0, 0.5, 0.3]))), C=C, V=V, softcap=rng.choice([0.0, 0.0, 30.0]),
                     smoothing=rng.choice([0.0, 0.0, 0.1]), z_weight=rng.choice([0.0, 1e-4]), weights=rng.choice(["mean", "rows"]), dtype=dtype)
    del case["name"]
    return case


# ------------------------------------------------------------------------------------------------ inputs

def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    dt = torch.float32 if case["dtype"] == "f32" else torch.bfloat16

    def normal(*shape, std=1.0):
        return (torch.randn(*shape, generator=gen, device="cuda") * std).to(dt)

    st = {"case": case}
    if case["kind"].startswith("rotate"):
        H, H_kv, d, rot = (case[n] for n in ("H", "H_kv", "d", "rot"))
        M = case["B"] if case["kind"] == "rotate_step" else case["M"]
        # the projection's result in one piece, as a fused projection leaves it
        qkv = normal(M, H + 2 * H_kv, d, std=1.3)
        st["Q"], st["K"], st["V"] = qkv[:, :H], qkv[:, H:H + H_kv], qkv[:, H + H_kv:]
        st["inv_freq"] = (500000.0 ** (-torch.arange(0, rot, 2, device="cuda", dtype=torch.float64) / rot)).float()
        st["eps"] = 1e-6
        for name, heads in (("w_q", H), ("w_k", H_kv)):
            shape = (heads, d) if case["per_head"] else (d,)
            st[name] = (1.0 + 0.2 * torch.randn(*shape, generator=gen, device="cuda")).to(dt) if case["norm"] != "none" else None
        if case["kind"] == "rotate_step":
            B, S = case["B"], case["S"]
            st["K_cache"], st["V_cache"] = normal(B, S, H_kv, d), normal(B, S, H_kv, d)
            st["lengths"] = torch.randint(1, S + 1, (B,), generator=gen, device="cuda", dtype=torch.int32)
            st["lengths"][0] = S
            return st
        st["positions"] = None
        if case["kept"]:  # of tokens far into a long context
            st["positions"] = torch.randint(0, 131072, (M,), generator=gen, device="cuda").sort().values.to(torch.int32)
        if case["kind"] == "rotate_grad":
            st["dQ_out"], st["dK_out"] = normal(M, H, d, std=0.05), normal(M, H_kv, d, std=0.05)
        return st
    S, M, C = case["S"], case["M"], case["C"]
    keep = torch.rand(S, generator=gen, device="cuda").topk(M).indices.sort().values.to(torch.int32)
    st["kept"] = keep if M < S else None
    if case["kind"] in ("drop", "drop_grad"):
        st["rng"] = torch.randint(-(1 << 62), 1 << 62, (2,), generator=gen, device="cuda", dtype=torch.int64)
        st["site"] = 5
        st["Y"] = normal(M, C, std=0.7)
        st["R"] = normal(S, C, std=2.0)
        return st
    V = case["V"]
    st["labels"] = torch.randint(0, V, (M,), generator=gen, device="cuda", dtype=torch.int32)
    st["W"] = normal(V, C, std=1.3 / math.sqrt(C))
    X = torch.randn(S, C, generator=gen, device="cuda")
    # tokens that the model expects more or less: their rows lean towards their labels' weights
    rows = keep.long() if M < S else torch.arange(S, device="cuda")
    X[rows] += torch.rand(M, 1, generator=gen, device="cuda") * 6 * st["W"][st["labels"].long()].float()
    st["X"] = X.to(dt)
    st["labels"][torch.rand(M, generator=gen, device="cuda") < 0.1] = -100  # a prompt's tokens have no label
    if case["kind"] == "loss_grad":
        loss, st["lse"], total = _loss_plain(st)
        st["dloss"] = total[3:] if case["weights"] == "mean" else torch.rand(M, generator=gen, device="cuda") / M
    return st


# ------------------------------------------------------------------------------------------------ the plain forms

def _turns(st, positions):
    """cos and sin of every position's angles [M, 1, rot / 2]: the angles in 64 bits, for far positions."""
    angle = positions.double().view(-1, 1, 1) * st["inv_freq"].double()
    return torch.cos(angle).float(), torch.sin(angle).float()


def _turned(x, cos, sin, pairs):
    """Rotates the first 2 * cos.shape[2] channels of every head of x [M, heads, d] (32 bits)."""
    rot = 2 * cos.shape[2]
    head, rest = x[:, :, :rot], x[:, :, rot:]
    if pairs:
        a, b = head[:, :, 0::2], head[:, :, 1::2]
        turned = torch.stack([a * cos - b * sin, b * cos + a * sin], dim=3).flatten(2)
    else:
        a, b = head[:, :, :rot // 2], head[:, :, rot // 2:]
        turned = torch.cat([a * cos - b * sin, b * cos + a * sin], dim=2)
    return torch.cat([turned, rest], dim=2)


def _normed(x, mode, eps):
    """x [M, heads, d] in 32 bits -> (normed before the weight, 1 / deviation)."""
    if mode == "none":
        return x, torch.ones_like(x[:, :, :1])
    x = x - x.mean(dim=2, keepdim=True) if mode == "layer" else x
    rstd = torch.rsqrt((x * x).mean(dim=2, keepdim=True) + eps)
    return x * rstd, rstd


def _positions(st):
    return st["positions"] if st["positions"] is not None else torch.arange(st["case"]["M"], device=st["Q"].device)


def _rotate_one(st, x, w, cos, sin):
    case = st["case"]
    y = _normed(x.float(), case["norm"], st["eps"])[0]
    y = y * w.float() if w is not None else y
    return _turned(y, cos, sin, case["pairs"]).to(x.dtype)


def _rotate_plain(st):
    cos, sin = _turns(st, _positions(st))
    return _rotate_one(st, st["Q"], st["w_q"], cos, sin), _rotate_one(st, st["K"], st["w_k"], cos, sin)


def _rotate_step_plain(st):
    cos, sin = _turns(st, st["lengths"] - 1)
    rows, at = torch.arange(st["case"]["B"], device=st["Q"].device), st["lengths"].long() - 1
    st["K_cache"][rows, at] = _rotate_one(st, st["K"], st["w_k"], cos, sin)
    st["V_cache"][rows, at] = st["V"]
    return _rotate_one(st, st["Q"], st["w_q"], cos, sin), st["K_cache"], st["V_cache"]


def _rotate_grad_one(st, dy, x, w, cos, sin):
    case = st["case"]
    t = _turned(dy.float(), cos, -sin, case["pairs"])  # the transposed rotation
    xhat, rstd = _normed(x.float(), case["norm"], st["eps"])
    if case["norm"] == "none":
        return t.to(x.dtype), None
    dw = (t * xhat).sum(dim=0 if case["per_head"] else (0, 1), dtype=torch.float64).float()
    t = t * w.float()
    dx = t - xhat * (t * xhat).mean(dim=2, keepdim=True)
    dx = dx - t.mean(dim=2, keepdim=True) if case["norm"] == "layer" else dx
    return (dx * rstd).to(x.dtype), dw


def _rotate_grad_plain(st):
    cos, sin = _turns(st, _positions(st))
    dQ, dw_q = _rotate_grad_one(st, st["dQ_out"], st["Q"], st["w_q"], cos, sin)
    dK, dw_k = _rotate_grad_one(st, st["dK_out"], st["K"], st["w_k"], cos, sin)
    return dQ, dK, dw_q, dw_k


_LOW = 0xffffffff


def _philox_round(c, k):
    """One round of Philox 4x32 (Salmon, Moraes, Dror, Shaw, 2011) on four 32-bit words held in 64 bits."""
    def product(a, b):  # high and low word of a * b, by halves of b: nothing passes 63 bits
        t, u = a * (b & 0xffff), a * (b >> 16)
        return (u + (t >> 16)) >> 16, (((u & 0xffff) << 16) + t) & _LOW

    hi0, lo0 = product(c[0], 0xD2511F53)
    hi1, lo1 = product(c[2], 0xCD9E8D57)
    return hi1 ^ c[1] ^ k[0], lo1, hi0 ^ c[3] ^ k[1], lo0


def _kept_mask(st, rows, C):
    """Which elements of the rows (token numbers) stay [M, C]: eight columns share one block of the generator, 16 bits each."""
    case, rng = st["case"], st["rng"]
    key = [rng[0] & _LOW, (rng[0] >> 32) & _LOW]
    stream = rng[1] + st["site"]
    groups = torch.arange(-(-C // 8), device=rows.device)
    shape = (len(rows), len(groups))
    c = (groups.expand(shape), rows.view(-1, 1).expand(shape), (stream & _LOW).expand(shape), ((stream >> 32) & _LOW).expand(shape))
    for _ in range(10):
        c = _philox_round(c, key)
        key = [(key[0] + 0x9E3779B9) & _LOW, (key[1] + 0xBB67AE85) & _LOW]
    bits = torch.stack([c[0] & 0xffff, c[0] >> 16, c[1] & 0xffff, c[1] >> 16, c[2] & 0xffff, c[2] >> 16, c[3] & 0xffff, c[3] >> 16], dim=2)
    return bits.flatten(1)[:, :C] < _keep16(case["p"])


def _keep16(p):
    return max(1, int(math.floor((1.0 - p) * 65536 + 0.5)))


def _rows(st):
    return st["kept"].long() if st["kept"] is not None else torch.arange(st["case"]["M"], device="cuda")


def _drop_plain(st):
    R, rows = st["R"], _rows(st)
    scale = 65536 / _keep16(st["case"]["p"])
    R[rows] = (R[rows].float() + torch.where(_kept_mask(st, rows, R.shape[1]), st["Y"].float() * scale, 0.0)).to(R.dtype)
    return R


def _drop_grad_plain(st):
    dR, rows = st["R"], _rows(st)
    scale = 65536 / _keep16(st["case"]["p"])
    return torch.where(_kept_mask(st, rows, dR.shape[1]), dR[rows].float() * scale, 0.0).to(dR.dtype)


def _logits(st):
    x = torch.matmul(st["X"][_rows(st)].float(), st["W"].float().t())
    cap = st["case"]["softcap"]
    return cap * torch.tanh(x / cap) if cap else x


def _labelled(st):
    labels = st["labels"].long()
    there = (labels >= 0) & (labels < st["case"]["V"])
    return there, labels.clamp(0, st["case"]["V"] - 1)


def _loss_plain(st):
    case = st["case"]
    x = _logits(st)
    there, at = _labelled(st)
    top = x.amax(dim=1, keepdim=True)
    lse = (top + torch.log(torch.exp(x - top).sum(dim=1, keepdim=True))).squeeze(1)
    s = case["smoothing"]
    loss = lse - (1 - s) * x.gather(1, at.view(-1, 1)).squeeze(1) + case["z_weight"] * lse * lse
    loss = loss - s * x.mean(dim=1) if s else loss
    loss = torch.where(there, loss, 0.0)
    n = there.sum().double()
    total = loss.double().sum()
    return loss, lse, torch.stack([total, n, total / n.clamp(min=1), 1 / n.clamp(min=1) * (n > 0)]).float()


def _loss_grad_plain(st):
    case, dt = st["case"], st["X"].dtype
    s, cap = case["smoothing"], case["softcap"]
    x = _logits(st)
    there, at = _labelled(st)
    lse = st["lse"].view(-1, 1)
    g = torch.exp(x - lse) * (1 + 2 * case["z_weight"] * lse) - s / case["V"]
    g.scatter_add_(1, at.view(-1, 1), torch.full_like(lse, s - 1))
    g = g * torch.where(there, st["dloss"], 0.0).view(-1, 1)
    g = g * (1 - (x / cap) ** 2) if cap else g
    return torch.matmul(g, st["W"].float()).to(dt), torch.matmul(g.t(), st["X"][_rows(st)].float()).to(dt)


# ------------------------------------------------------------------------------------------------ the framework's calls

def _run_own(st):
    from paper_2501_09767_amd import lemo

    case = st["case"]
    kind = case["kind"]
    if kind.startswith("rotate"):
        how = dict(norm={"none": lemo.NORM_NONE, "rms": lemo.NORM_RMS, "layer": lemo.NORM_LAYER}[case["norm"]], w_q=st["w_q"], w_k=st["w_k"], eps=st["eps"],
                   flags=lemo.ROTATE_PAIRS if case["pairs"] else 0)
        if kind == "rotate":
            return lemo.lemo_qk_rotate(st["Q"], st["K"], st["inv_freq"], st["positions"], **how)
        if kind == "rotate_grad":
            return tuple(lemo.lemo_qk_rotate_grad(st["dQ_out"], st["dK_out"], st["Q"], st["K"], st["inv_freq"], st["positions"], **how))
        Q = lemo.lemo_qk_rotate_step(st["Q"], st["K"], st["V"], st["K_cache"], st["V_cache"], st["lengths"], st["inv_freq"], **how)
        return Q, st["K_cache"], st["V_cache"]
    if kind == "drop":
        return lemo.lemo_dropout_add(st["Y"], st["R"], st["kept"], st["rng"], case["p"], st["site"])
    if kind == "drop_grad":
        return lemo.lemo_dropout_add_grad(st["R"], st["kept"], st["rng"], case["p"], st["site"])
    how = dict(softcap=case["softcap"], smoothing=case["smoothing"], z_weight=case["z_weight"])
    if kind == "loss":
        return tuple(lemo.lemo_vocab_loss(st["X"], st["kept"], st["W"], st["labels"], **how))
    return tuple(lemo.lemo_vocab_loss_grad(st["dloss"], st["X"], st["kept"], st["W"], st["labels"], st["lse"], **how))


def run(st):
    if own:
        return _run_own(st)
    return {"rotate": _rotate_plain, "rotate_grad": _rotate_grad_plain, "rotate_step": _rotate_step_plain, "drop": _drop_plain,
            "drop_grad": _drop_grad_plain, "loss": _loss_plain, "loss_grad": _loss_grad_plain}[st["case"]["kind"]](st)


# ------------------------------------------------------------------------------------------------ what a pass cannot do without

def work(case):
    kind, e = case["kind"], 4 if case["dtype"] == "f32" else 2
    if kind.startswith("rotate"):
        heads, d = case["H"] + case["H_kv"], case["d"]
        if kind == "rotate_step":
            n = case["B"] * d
            return {"bytes": 2 * e * n * (heads + case["H_kv"]) + 4 * case["B"], "flops": 8 * n * heads}
        n = case["M"] * heads * d
        places = 4 * case["M"] if case["kept"] else 0
        return {"bytes": (2 if kind == "rotate" else 3) * e * n + places, "flops": (8 if kind == "rotate" else 16) * n}
    M, C = case["M"], case["C"]
    if kind == "drop":
        return {"bytes": 3 * e * M * C + 4 * M, "flops": 2 * M * C}
    if kind == "drop_grad":
        return {"bytes": 2 * e * M * C + 4 * M, "flops": M * C}
    V = case["V"]
    if kind == "loss":
        return {"bytes": e * C * (M + V) + 16 * M, "flops": 2 * M * C * V}
    # the logits once more, then two products
    return {"bytes": 2 * e * C * (M + V) + 16 * M, "flops": 6 * M * C * V}


# ------------------------------------------------------------------------------------------------ the definition in 64 bits

def exact(case, seed):
    """From the definitions, in 64 bits: rotations as products of complex numbers, gradients of norms by autograd, the loss by rows."""
    st = prepare(case, seed)
    if case["kind"].startswith("rotate"):
        return _rotate_exact(st)
    if case["kind"] in ("drop", "drop_grad"):
        return _drop_exact(st)
    return _loss_exact(st)


def _rotate_exact(st):
    case, rot, d = st["case"], st["case"]["rot"], st["case"]["d"]
    place = st["lengths"].double() - 1 if case["kind"] == "rotate_step" else _positions(st).double()
    angle = place[:, None] * st["inv_freq"].double()[None]
    unit = torch.polar(torch.ones_like(angle), angle)[:, None]
    n = torch.arange(rot // 2, device="cuda")
    first, second = (2 * n, 2 * n + 1) if case["pairs"] else (n, n + rot // 2)

    def one(x, w):
        if case["norm"] == "layer":
            x = x - x.mean(dim=2, keepdim=True)
        if case["norm"] != "none":
            x = x / (x.square().sum(dim=2, keepdim=True) / d + st["eps"]).sqrt() * w
        z = torch.complex(x[:, :, first], x[:, :, second]) * unit
        order = torch.cat([first, second, torch.arange(rot, d, device="cuda")]).argsort()
        return torch.cat([z.real, z.imag, x[:, :, rot:]], dim=2)[:, :, order]

    def wide(name):
        return None if st[name] is None else st[name].double().requires_grad_(case["kind"] == "rotate_grad")

    Q, K, w_q, w_k = wide("Q"), wide("K"), wide("w_q"), wide("w_k")
    Q_out, K_out = one(Q, w_q), one(K, w_k)
    if case["kind"] == "rotate":
        return Q_out, K_out
    if case["kind"] == "rotate_step":
        K_cache, V_cache = st["K_cache"].double(), st["V_cache"].double()
        rows, at = torch.arange(case["B"], device="cuda"), st["lengths"].long() - 1
        K_cache[rows, at], V_cache[rows, at] = K_out, st["V"].double()
        return Q_out, K_cache, V_cache
    back = torch.autograd.grad([Q_out, K_out], [t for t in (Q, K, w_q, w_k) if t is not None], [st["dQ_out"].double(), st["dK_out"].double()])
    return back if w_q is not None else (*back, None, None)


def _drop_exact(st):
    """The generator in Python's own integers for every word at once: numpy's 64-bit products of 32-bit words."""
    import numpy as np

    case, low = st["case"], np.uint64(_LOW)
    C, rows = case["C"], _rows(st).cpu().numpy().astype(np.uint64)
    seed, stream = (int(v) & 0xffffffffffffffff for v in st["rng"].tolist())
    stream = (stream + st["site"]) & 0xffffffffffffffff
    out = np.empty((len(rows), -(-C // 8), 8), dtype=np.uint16)
    step = max(1, (1 << 22) // (out.shape[1] or 1))
    for i in range(0, len(rows), step):
        part = rows[i:i + step]
        x0, x1 = np.broadcast_arrays(np.arange(out.shape[1], dtype=np.uint64)[None, :], part[:, None])
        x2, x3 = np.full_like(x0, stream & _LOW), np.full_like(x0, stream >> 32)
        for r in range(10):
            k0, k1 = np.uint64((seed + r * 0x9E3779B9) & _LOW), np.uint64(((seed >> 32) + r * 0xBB67AE85) & _LOW)
            p, q = x0 * np.uint64(0xD2511F53), x2 * np.uint64(0xCD9E8D57)
            x0, x1, x2, x3 = (q >> np.uint64(32)) ^ x1 ^ k0, q & low, (p >> np.uint64(32)) ^ x3 ^ k1, p & low
        out[i:i + step] = np.stack([x0, x1, x2, x3], axis=2).astype(np.uint32).view(np.uint16).reshape(len(part), -1, 8)
    keep = torch.from_numpy(out.reshape(len(rows), -1)[:, :C].astype(np.int32)).cuda() < _keep16(case["p"])
    factor = keep.double() * 65536 / _keep16(case["p"])
    R = st["R"].double()
    if case["kind"] == "drop_grad":
        return R[_rows(st)] * factor
    R[_rows(st)] += st["Y"].double() * factor
    return R


def _loss_exact(st):
    case = st["case"]
    V, s, z, cap = case["V"], case["smoothing"], case["z_weight"], case["softcap"]
    X, W = st["X"][_rows(st)].double(), st["W"].double()
    labels = st["labels"].long()
    losses, lses, dX, dW = [], [], [], torch.zeros_like(W) if case["kind"] == "loss_grad" else None
    for i in range(0, case["M"], 512):
        part = slice(i, min(case["M"], i + 512))
        x = X[part] @ W.t()
        u = cap * torch.tanh(x / cap) if cap else x
        ok = (labels[part] >= 0) & (labels[part] < V)
        hot = torch.zeros_like(x)
        hot[ok, labels[part][ok]] = 1.0
        want = (1 - s) * hot + s / V
        lse = torch.logsumexp(u, dim=1)
        if case["kind"] == "loss":
            lses.append(lse)
            losses.append(((lse + z * lse ** 2) - (want * u).sum(dim=1)) * ok)
            continue
        weight = st["dloss"].double().expand(case["M"])[part] * ok
        g = (torch.softmax(u, dim=1) * (1 + 2 * z * lse)[:, None] - want) * weight[:, None]
        if cap:
            g = g / torch.cosh(x / cap) ** 2
        dX.append(g @ W)
        dW += g.t() @ X[part]
    if case["kind"] == "loss_grad":
        return torch.cat(dX), dW
    loss, n = torch.cat(losses), int(((labels >= 0) & (labels < V)).sum())
    total = float(loss.sum())
    return loss, torch.cat(lses), torch.tensor([total, n, total / max(n, 1), 1.0 / n if n else 0.0], dtype=torch.float64)

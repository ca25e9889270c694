"""The operators around attention that are timed, over the sizes they are used at.

Attention (forward and backward), the norm of queries and keys for each head
with the rotary rotation (forward and backward), and dropout from a
counter-based generator with the residual sum (forward and backward).

``listed()`` gives the cases, ``draw(rng)`` one more of the same ranges,
``prepare(case, seed)`` what a program holds before the call, ``run(state)``
one pass (the plain form in fp32 torch where ``own`` is false, the public entry
points where it is true), ``exact(case, seed)`` the same outputs from the
definitions in 64 bits and ``work(case)`` the bytes and operations a pass
cannot do without.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

DEV = "cuda:0"
EPS = 1e-6


def listed():
    return [
        # the residual stream of an 8192-wide layer over 8192 tokens: a block's
        # output is dropped out and added to its input
        dict(name="dropout_residual_8192x8192_f32", kind="dropout", dir="fwd", M=8192, N=8192, dtype="f32",
             residual=True, p=0.1),
        # the smallest call, an odd width, the gradient's form: launch latency
        dict(name="dropout_bwd_509x383_bf16", kind="dropout", dir="bwd", M=509, N=383, dtype="bf16",
             residual=False, p=0.25),
        # queries and keys of an ordinary training batch, four queries to a key head
        dict(name="qk_norm_rope_4x4096_32_8_128_bf16", kind="rope", dir="fwd", B=4, T=4096, HQ=32, HK=8, D=128,
             R=128, x="bf16", y="bf16", interleaved=False),
        # a step of serving: one token of each of 64 sequences, from fp32 projections to a bf16 cache
        dict(name="qk_norm_rope_token_64x1_32_8_128", kind="rope", dir="fwd", B=64, T=1, HQ=32, HK=8, D=128,
             R=128, x="f32", y="bf16", interleaved=False),
        # the gradient, with both norms' weights, odd length, pairs side by side, half of each head rotated
        dict(name="qk_norm_rope_bwd_8x1021_16_16_64_f32", kind="rope", dir="bwd", B=8, T=1021, HQ=16, HK=16, D=64,
             R=32, x="f32", y="f32", interleaved=True),
        # a training batch's causal attention, forward
        dict(name="attention_4x4096_32_8_128_causal_bf16", kind="attn", dir="fwd", B=4, TQ=4096, TK=4096, HQ=32,
             HK=8, D=128, causal=True, dtype="bf16", lens="full"),
        # attention to another, shorter sequence of ragged length (odd sizes, one batch without a key), fp32
        dict(name="attention_8x509x383_8_8_64_ragged_f32", kind="attn", dir="fwd", B=8, TQ=509, TK=383, HQ=8, HK=8,
             D=64, causal=False, dtype="f32", lens="ragged"),
        # a step of serving: one token a sequence against caches of up to 8192 tokens
        dict(name="attention_token_16x1x8192_32_8_128_bf16", kind="attn", dir="fwd", B=16, TQ=1, TK=8192, HQ=32,
             HK=8, D=128, causal=True, dtype="bf16", lens="ragged"),
        # one long prompt
        dict(name="attention_1x16384_16_4_128_causal_bf16", kind="attn", dir="fwd", B=1, TQ=16384, TK=16384, HQ=16,
             HK=4, D=128, causal=True, dtype="bf16", lens="full"),
        # the training batch's gradient
        dict(name="attention_bwd_4x4096_32_8_128_causal_bf16", kind="attn", dir="bwd", B=4, TQ=4096, TK=4096, HQ=32,
             HK=8, D=128, causal=True, dtype="bf16", lens="full"),
        # the gradient in fp32, narrower heads
        dict(name="attention_bwd_4x1024_16_16_64_causal_f32", kind="attn", dir="bwd", B=4, TQ=1024, TK=1024, HQ=16,
             HK=16, D=64, causal=True, dtype="f32", lens="full"),
        # the gradient of a padded batch: odd and ragged lengths, a head width between two powers of two
        dict(name="attention_bwd_6x777_12_4_96_ragged_bf16", kind="attn", dir="bwd", B=6, TQ=777, TK=777, HQ=12,
             HK=4, D=96, causal=True, dtype="bf16", lens="ragged"),
    ]


def _size(rng, lo, hi):
    """A size from lo to hi, spread over its logarithm; multiples of 64 or 8 about as often as any."""
    v = math.exp(rng.uniform(math.log(lo), math.log(hi + 1)))
    g = rng.choice([64, 64, 8, 1])
    n = int(min(hi, max(lo, round(v / g) * g)))
    return n - 1 if n == 3072 else n


def draw(rng):
    kind = rng.choice(["dropout", "rope", "attn", "attn", "attn"])
    if kind == "dropout":
        fwd = rng.random() < 0.5
        return dict(kind=kind, dir="fwd" if fwd else "bwd", M=_size(rng, 1, 8192), N=_size(rng, 64, 8192),
                    dtype=rng.choice(["f32", "bf16"]), residual=fwd and rng.random() < 0.7,
                    p=rng.choice([0.05, 0.1, 0.25, 0.5]))
    heads = rng.choice([(32, 8), (16, 16), (16, 4), (12, 4), (8, 8), (8, 1), (7, 7)])
    D = rng.choice([64, 128, 128, 32, 80, 96, 112])
    if kind == "rope":
        fwd = rng.random() < 0.5
        x, y = rng.choice([("f32", "f32"), ("bf16", "bf16"), ("f32", "bf16")])
        T = 1 if fwd and rng.random() < 0.3 else _size(rng, 16, 4096)
        B = max(1, min(64 if T == 1 else 16, 16384 // T, _size(rng, 1, 64)))
        return dict(kind=kind, dir="fwd" if fwd else "bwd", B=B, T=T, HQ=heads[0], HK=heads[1], D=D,
                    R=rng.choice([D, D, D // 2]), x=x, y=y, interleaved=rng.random() < 0.4)
    dtype = rng.choice(["bf16", "bf16", "f32"])
    case = dict(kind=kind, HQ=heads[0], HK=heads[1], D=D, dtype=dtype)
    form = rng.choice(["train", "train", "train", "cross", "token"])
    if form == "token":
        TK = _size(rng, 16, 16384)
        case.update(dir="fwd", TQ=1, TK=TK, B=max(1, min(16, 131072 // TK, _size(rng, 1, 16))), causal=True,
                    lens="ragged")
    else:
        fwd = rng.random() < 0.5
        TK = _size(rng, 64, 8192 if fwd and dtype == "bf16" else 4096 if dtype == "bf16" else 2048)
        TQ = TK if form == "train" else _size(rng, 16, TK)
        cap = (4 * 4096 * 4096 * 32 if dtype == "bf16" else 4 * 1024 * 1024 * 32) // 2
        B = max(1, min(16, cap // (TQ * TK * heads[0]), _size(rng, 1, 16)))
        case.update(dir="fwd" if fwd else "bwd", TQ=TQ, TK=TK, B=B, causal=form == "train",
                    lens=rng.choice(["full", "ragged"]))
    return case


# ------------------------------------------------------------------ inputs
_DT = {"f32": torch.float32, "bf16": torch.bfloat16}


def _normal(g, shape, dtype):
    return torch.randn(shape, generator=g, device=DEV).to(_DT[dtype])


def _gen(seed):
    g = torch.Generator(DEV)
    g.manual_seed(seed)
    return g


def prepare(case, seed):
    s = _INPUTS[case["kind"]](case, seed)
    s["case"] = case
    if own:
        _buffers(s)
    return s


def _dropout_inputs(case, seed):
    g = _gen(seed)
    s = dict(x=_normal(g, (case["M"], case["N"]), case["dtype"]), p=case["p"], seed=1234567890123 + seed,
             offset=(1 << 33) + 977 * seed)
    s["residual"] = _normal(g, (case["M"], case["N"]), case["dtype"]) if case["residual"] else None
    return s


def _rope_inputs(case, seed):
    g = _gen(seed)
    B, T, HQ, HK, D, R = (case[k] for k in ("B", "T", "HQ", "HK", "D", "R"))
    # views of the packed projection, as a layer's output holds them
    qkv = _normal(g, (B, T, (HQ + 2 * HK) * D), case["x"])
    s = dict(q=qkv[..., :HQ * D].unflatten(-1, (HQ, D)), k=qkv[..., HQ * D:(HQ + HK) * D].unflatten(-1, (HK, D)))
    s["wq"] = 1 + 0.1 * torch.randn(D, generator=g, device=DEV)
    s["wk"] = 1 + 0.1 * torch.randn(D, generator=g, device=DEV)
    if T == 1:  # every sequence at a position of its own
        pos = torch.randint(0, 8192, (B, 1), generator=g, device=DEV).double()
    else:
        pos = torch.arange(T, device=DEV).double()[None]
    ang = pos[..., None] * 10000.0 ** (-torch.arange(0, R, 2, device=DEV).double() / R)
    s["cos"], s["sin"] = (f(ang).float().expand(B, T, R // 2) for f in (torch.cos, torch.sin))
    if case["dir"] == "bwd":
        s["dyq"] = _normal(g, (B, T, HQ, D), case["y"])
        s["dyk"] = _normal(g, (B, T, HK, D), case["y"])
    return s


def _attn_inputs(case, seed):
    g = _gen(seed)
    B, TQ, TK, HQ, HK, D = (case[k] for k in ("B", "TQ", "TK", "HQ", "HK", "D"))
    s = dict(q=_normal(g, (B, TQ, HQ, D), case["dtype"]), k=_normal(g, (B, TK, HK, D), case["dtype"]),
             v=_normal(g, (B, TK, HK, D), case["dtype"]), kv_len=None)
    if case["lens"] == "ragged":
        n = torch.randint(TK // 4, TK + 1, (B,), generator=g, device=DEV)
        if TQ > 1:
            n[B // 2] = 0 if B > 1 else TK // 2
        s["kv_len"] = n.to(torch.int32)
    if case["dir"] == "bwd":
        s["do"] = _normal(g, (B, TQ, HQ, D), case["dtype"])
        s["case"] = case
        s["o"], s["lse"] = _attn_fwd(s)
    return s


_INPUTS = {"dropout": _dropout_inputs, "rope": _rope_inputs, "attn": _attn_inputs}


# ------------------------------------------------------- the plain forms
def run(s):
    case = s["case"]
    table = _OWN if own else _PLAIN
    return table[case["kind"], case["dir"]](s)


_M32 = 0xFFFFFFFF


def _philox(counter, seed):
    """The four 32-bit words of the 10-round generator at 64-bit counters (int64 tensors)."""
    x0, x1 = counter & _M32, (counter >> 32) & _M32
    x2, x3 = torch.zeros_like(x0), torch.zeros_like(x0)
    k0, k1 = seed & _M32, (seed >> 32) & _M32
    for _ in range(10):
        a, b = x0 * 0xD2511F53, x2 * 0xCD9E8D57  # the low 64 bits, whatever the sign
        x0, x1, x2, x3 = (((b >> 32) & _M32) ^ x1 ^ k0, b & _M32, ((a >> 32) & _M32) ^ x3 ^ k1, a & _M32)
        k0, k1 = (k0 + 0x9E3779B9) & _M32, (k1 + 0xBB67AE85) & _M32
    return x0, x1, x2, x3


def _keep(x, p, seed, offset):
    """(which elements stay, the scale of those): element i takes the 16 bits i % 8 of the words at
    counter offset + i // 8 and stays where they are p's 65536ths or more."""
    n = x.numel()
    words = _philox(torch.arange((n + 7) // 8, device=x.device) + offset, seed)
    halves = torch.stack([h for w in words for h in (w & 0xFFFF, w >> 16)], dim=1)
    drop = round(p * 65536)
    return (halves.flatten()[:n] >= drop).view_as(x), 65536.0 / (65536 - drop) if drop < 65536 else 0.0


def _dropout(s):
    x = s["x"]
    keep, scale = _keep(x, s["p"], s["seed"], s["offset"])
    y = torch.where(keep, x.float() * scale, 0.0)
    if s["residual"] is not None:
        y = y + s["residual"].float()
    return y.to(x.dtype)


def _pairs(x, R, interleaved):
    return (x[..., 0:R:2], x[..., 1:R:2]) if interleaved else (x[..., :R // 2], x[..., R // 2:R])


def _unpairs(a, b, rest, interleaved):
    head = torch.stack([a, b], dim=-1).flatten(-2) if interleaved else torch.cat([a, b], dim=-1)
    return torch.cat([head, rest], dim=-1)


def _norm_rope(x, w, cos, sin, inter, dtype):
    R = 2 * cos.shape[-1]
    x = x.float()
    n = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS) * w
    a, b = _pairs(n, R, inter)
    c, t = cos[:, :, None], sin[:, :, None]
    return _unpairs(a * c - b * t, b * c + a * t, n[..., R:], inter).to(dtype)


def _rope_fwd(s):
    case = s["case"]
    dt = _DT[case["y"]]
    return [_norm_rope(s["q"], s["wq"], s["cos"], s["sin"], case["interleaved"], dt),
            _norm_rope(s["k"], s["wk"], s["cos"], s["sin"], case["interleaved"], dt)]


def _norm_rope_grad(x, w, cos, sin, dy, inter):
    R = 2 * cos.shape[-1]
    dt = dy.dtype
    x, dy = x.float(), dy.float()
    r = torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS)
    n = x * r
    a, b = _pairs(dy, R, inter)
    c, t = cos[:, :, None], sin[:, :, None]
    g = _unpairs(a * c + b * t, b * c - a * t, dy[..., R:], inter)
    dw = (g * n).flatten(0, 2).sum(0)
    dn = g * w
    return (r * (dn - n * (n * dn).mean(-1, keepdim=True))).to(dt), dw


def _rope_bwd(s):
    inter = s["case"]["interleaved"]
    dq, dwq = _norm_rope_grad(s["q"], s["wq"], s["cos"], s["sin"], s["dyq"], inter)
    dk, dwk = _norm_rope_grad(s["k"], s["wk"], s["cos"], s["sin"], s["dyk"], inter)
    return [dq, dk, dwq, dwk]


def _banned(s):
    """[B, 1, TQ, TK] (or a broadcast of it): true where a query may not see a key; None if all may."""
    case = s["case"]
    ban = None
    j = torch.arange(case["TK"], device=DEV)
    if case["causal"]:
        i = torch.arange(case["TQ"], device=DEV) + case["TK"] - case["TQ"]
        ban = (j[None] > i[:, None])[None, None]
    if s["kv_len"] is not None:
        far = j[None, None, None] >= s["kv_len"][:, None, None, None]
        ban = far if ban is None else ban | far
    return ban


def _grouped(x, HK):
    """[B, T, H, D] -> [B * HK, (H / HK) * T, D], fp32 and contiguous: the query heads of a key head together."""
    B, T, H, D = x.shape
    return x.float().view(B, T, HK, H // HK, D).permute(0, 2, 3, 1, 4).reshape(B * HK, H // HK * T, D)


def _ungrouped(x, B, T, HK):
    G, D = x.shape[1] // T, x.shape[2]
    return x.view(B, HK, G, T, D).permute(0, 3, 1, 2, 4).reshape(B, T, HK * G, D)


def _scores(s, q, k):
    """[B, HQ, TQ, TK] scaled scores, -inf where banned."""
    case = s["case"]
    S = torch.bmm(q, k.transpose(1, 2).contiguous()).mul_(case["D"] ** -0.5)
    S = S.view(case["B"], case["HQ"], case["TQ"], case["TK"])
    ban = _banned(s)
    return S if ban is None else S.masked_fill_(ban, -math.inf)


def _attn_fwd(s):
    case = s["case"]
    B, TQ, TK, HQ, HK = (case[c] for c in ("B", "TQ", "TK", "HQ", "HK"))
    S = _scores(s, _grouped(s["q"], HK), _grouped(s["k"], HK))
    m = S.amax(-1, keepdim=True)
    P = S.sub_(torch.where(m == -math.inf, 0.0, m)).exp_()
    total = P.sum(-1, keepdim=True)
    o = torch.bmm(P.view(B * HK, -1, TK), _grouped(s["v"], HK)).view(B, HQ, TQ, -1)
    o = torch.where(total > 0, o / total, 0.0)
    o = _ungrouped(o.view(B * HK, -1, case["D"]), B, TQ, HK)
    return [o.to(s["q"].dtype), (m + total.log()).squeeze(-1)]


def _attn_bwd(s):
    case = s["case"]
    B, TQ, TK, HQ, HK, D = (case[c] for c in ("B", "TQ", "TK", "HQ", "HK", "D"))
    q, k, v, do = (_grouped(s[n], HK) for n in ("q", "k", "v", "do"))
    lse = s["lse"][..., None]
    P = _scores(s, q, k).sub_(torch.where(lse == -math.inf, 0.0, lse)).exp_().view(B * HK, -1, TK)
    dv = torch.bmm(P.transpose(1, 2), do)
    delta = (do * _grouped(s["o"], HK)).sum(-1, keepdim=True)
    dS = torch.bmm(do, v.transpose(1, 2).contiguous()).sub_(delta).mul_(P).mul_(D ** -0.5)
    dq = torch.bmm(dS, k)
    dk = torch.bmm(dS.transpose(1, 2), q)
    dt = s["q"].dtype
    return [_ungrouped(dq, B, TQ, HK).to(dt), _ungrouped(dk, B, TK, HK).to(dt), _ungrouped(dv, B, TK, HK).to(dt)]


_PLAIN = {("dropout", "fwd"): _dropout, ("dropout", "bwd"): _dropout, ("rope", "fwd"): _rope_fwd,
          ("rope", "bwd"): _rope_bwd, ("attn", "fwd"): _attn_fwd, ("attn", "bwd"): _attn_bwd}


# ------------------------------------------------- the framework's calls
def _workspace(n):
    return torch.empty(n, dtype=torch.uint8, device=DEV) if n else None


def _buffers(s):
    """Output buffers and workspace, as a training loop or a server keeps them."""
    from paper_2602_00125_amd import binding as mt

    s["mt"] = mt
    case = s["case"]
    if case["kind"] == "dropout":
        s["y"] = torch.empty_like(s["x"])
    elif case["kind"] == "rope":
        s["yq"], s["yk"] = (torch.empty(s[n].shape, dtype=_DT[case["y"]], device=DEV) for n in ("q", "k"))
        if case["dir"] == "bwd":
            s["dwq"], s["dwk"] = torch.empty_like(s["wq"]), torch.empty_like(s["wk"])
            s["ws"] = _workspace(mt.qk_norm_rope_bwd_workspace(s["q"], s["k"], s["wq"], s["wk"], s["cos"], s["sin"],
                                                               s["dyq"], s["dyk"], s["yq"], s["yk"], s["dwq"],
                                                               s["dwk"]))
    elif case["dir"] == "fwd":
        s["o"] = torch.empty_like(s["q"])
        s["lse"] = torch.empty(case["B"], case["HQ"], case["TQ"], device=DEV)
        s["ws"] = _workspace(mt.attention_fwd_workspace(s["q"], s["k"], s["v"], s["o"], s["lse"], kv_len=s["kv_len"],
                                                        causal=case["causal"]))
    else:
        s["dq"], s["dk"], s["dv"] = (torch.empty_like(s[n]) for n in ("q", "k", "v"))
        s["ws"] = _workspace(mt.attention_bwd_workspace(s["q"], s["k"], s["v"], s["o"], s["lse"], s["do"], s["dq"],
                                                        s["dk"], s["dv"], kv_len=s["kv_len"],
                                                        causal=case["causal"]))


def _own_dropout_fwd(s):
    s["mt"].dropout_fwd(s["x"], s["residual"], s["p"], s["seed"], s["offset"], s["y"])
    return s["y"]


def _own_dropout_bwd(s):
    s["mt"].dropout_bwd(s["x"], s["p"], s["seed"], s["offset"], s["y"])
    return s["y"]


def _own_rope_fwd(s):
    s["mt"].qk_norm_rope_fwd(s["q"], s["k"], s["wq"], s["wk"], s["cos"], s["sin"], s["yq"], s["yk"], eps=EPS,
                             interleaved=s["case"]["interleaved"])
    return [s["yq"], s["yk"]]


def _own_rope_bwd(s):
    s["mt"].qk_norm_rope_bwd(s["q"], s["k"], s["wq"], s["wk"], s["cos"], s["sin"], s["dyq"], s["dyk"], s["yq"],
                             s["yk"], s["dwq"], s["dwk"], eps=EPS, interleaved=s["case"]["interleaved"],
                             workspace=s["ws"])
    return [s["yq"], s["yk"], s["dwq"], s["dwk"]]


def _own_attn_fwd(s):
    s["mt"].attention_fwd(s["q"], s["k"], s["v"], s["o"], s["lse"], kv_len=s["kv_len"], causal=s["case"]["causal"],
                          workspace=s["ws"])
    return [s["o"], s["lse"]]


def _own_attn_bwd(s):
    s["mt"].attention_bwd(s["q"], s["k"], s["v"], s["o"], s["lse"], s["do"], s["dq"], s["dk"], s["dv"],
                          kv_len=s["kv_len"], causal=s["case"]["causal"], workspace=s["ws"])
    return [s["dq"], s["dk"], s["dv"]]


_OWN = {("dropout", "fwd"): _own_dropout_fwd, ("dropout", "bwd"): _own_dropout_bwd, ("rope", "fwd"): _own_rope_fwd,
        ("rope", "bwd"): _own_rope_bwd, ("attn", "fwd"): _own_attn_fwd, ("attn", "bwd"): _own_attn_bwd}


# ------------------------------------------------------------- 64 bits
def exact(case, seed):
    s = _INPUTS[case["kind"]](case, seed)
    s["case"] = case
    return _EXACT[case["kind"], case["dir"]](s)


def _exact_dropout(s):
    """Element by element: the generator in numpy's unsigned integers."""
    n = s["x"].numel()
    u = np.uint64
    low, shift = u(_M32), u(32)
    ctr = np.arange((n + 7) // 8, dtype=np.uint64) + u(s["offset"])
    w = [ctr & low, ctr >> shift, np.zeros_like(ctr), np.zeros_like(ctr)]
    key = [s["seed"] % 2**32, s["seed"] >> 32]
    for _ in range(10):
        a, b = w[0] * u(0xD2511F53), w[2] * u(0xCD9E8D57)
        w = [(b >> shift) ^ w[1] ^ u(key[0]), b & low, (a >> shift) ^ w[3] ^ u(key[1]), a & low]
        key = [(key[0] + 0x9E3779B9) % 2**32, (key[1] + 0xBB67AE85) % 2**32]
    # the words' halves in order are their little-endian 16-bit pieces
    draws = np.stack(w, 1).astype("<u4").view("<u2").reshape(-1)[:n]
    drop = int(s["p"] * 65536 + 0.5)
    factor = torch.from_numpy((draws >= drop).astype(np.float64) * (65536 / (65536 - drop))).to(DEV)
    y = s["x"].double() * factor.view(s["x"].shape)
    return y if s["residual"] is None else y + s["residual"].double()


def _exact_rotation(cos, sin, D, inter):
    """[B, T, D / 2...] as complex factors over pair indices: (indices of first, of second, factor)."""
    R = 2 * cos.shape[-1]
    i = torch.arange(R // 2, device=DEV)
    first, second = (2 * i, 2 * i + 1) if inter else (i, i + R // 2)
    return first, second, torch.complex(cos.double(), sin.double())[:, :, None]


def _exact_rotate(x, rot, conj):
    first, second, f = rot
    z = torch.complex(x[..., first], x[..., second]) * (f.conj() if conj else f)
    y = x.clone()
    y[..., first], y[..., second] = z.real, z.imag
    return y


def _exact_rope_fwd(s):
    out = []
    for x, w in ((s["q"], s["wq"]), (s["k"], s["wk"])):
        x = x.double()
        n = x / torch.sqrt(x.square().sum(-1, keepdim=True) / x.shape[-1] + EPS)
        rot = _exact_rotation(s["cos"], s["sin"], x.shape[-1], s["case"]["interleaved"])
        out.append(_exact_rotate(n * w.double(), rot, False))
    return out


def _exact_rope_bwd(s):
    dx, dw = [], []
    for x, w, dy in ((s["q"], s["wq"], s["dyq"]), (s["k"], s["wk"], s["dyk"])):
        x, D = x.double(), x.shape[-1]
        ms = x.square().sum(-1, keepdim=True) / D + EPS
        g = _exact_rotate(dy.double(), _exact_rotation(s["cos"], s["sin"], D, s["case"]["interleaved"]), True)
        dw.append((g * x / ms.sqrt()).sum((0, 1, 2)))
        gw = g * w.double()
        # d(x / sqrt(ms)) = gw / sqrt(ms) - x (x . gw) / (D ms^(3/2))
        dx.append(gw / ms.sqrt() - x * (x * gw).sum(-1, keepdim=True) / (D * ms ** 1.5))
    return dx + dw


def _exact_heads(s):
    """For each (batch, query head): its index, its key head, fp64 q, k, v and the visible keys of each query."""
    case = s["case"]
    G = case["HQ"] // case["HK"]
    i = torch.arange(case["TQ"], device=DEV)[:, None] + (case["TK"] - case["TQ"])
    for b in range(case["B"]):
        n = case["TK"] if s["kv_len"] is None else int(s["kv_len"][b])
        j = torch.arange(n, device=DEV)[None]
        seen = (j <= i) if case["causal"] else torch.ones(case["TQ"], n, dtype=torch.bool, device=DEV)
        for h in range(case["HQ"]):
            yield b, h, h // G, s["q"][b, :, h].double(), s["k"][b, :n, h // G].double(), \
                s["v"][b, :n, h // G].double(), seen


def _exact_probabilities(case, q, k, seen):
    """Softmax over the visible keys (zero rows where there are none) and its log-sum-exp."""
    z = torch.where(seen, q @ k.T / math.sqrt(case["D"]), -math.inf)
    lse = torch.logsumexp(z, dim=-1)
    return torch.exp(z - lse.clamp_min(-1e300)[:, None]), lse


def _exact_attn_fwd(s):
    case = s["case"]
    o = torch.zeros(s["q"].shape, dtype=torch.float64, device=DEV)
    lses = torch.full((case["B"], case["HQ"], case["TQ"]), -math.inf, dtype=torch.float64, device=DEV)
    for b, h, _, q, k, v, seen in _exact_heads(s):
        if len(k):
            P, lses[b, h] = _exact_probabilities(case, q, k, seen)
            o[b, :, h] = P @ v
    return [o, lses]


def _exact_attn_bwd(s):
    """The gradients of <do, attention(q, k, v)> with respect to q, k and v."""
    case = s["case"]
    dq, dk, dv = (torch.zeros(s[n].shape, dtype=torch.float64, device=DEV) for n in ("q", "k", "v"))
    for b, h, hk, q, k, v, seen in _exact_heads(s):
        if not len(k):
            continue
        P, _ = _exact_probabilities(case, q, k, seen)
        do = s["do"][b, :, h].double()
        dP = do @ v.T
        dz = P * (dP - (P * dP).sum(-1, keepdim=True)) / math.sqrt(case["D"])
        dq[b, :, h] = dz @ k
        dk[b, :len(k), hk] += dz.T @ q
        dv[b, :len(k), hk] += P.T @ do
    return [dq, dk, dv]


_EXACT = {("dropout", "fwd"): _exact_dropout, ("dropout", "bwd"): _exact_dropout, ("rope", "fwd"): _exact_rope_fwd,
          ("rope", "bwd"): _exact_rope_bwd, ("attn", "fwd"): _exact_attn_fwd, ("attn", "bwd"): _exact_attn_bwd}


# ---------------------------------------------------------------- work
def work(case):
    size = {"f32": 4, "bf16": 2}
    if case["kind"] == "dropout":
        n = case["M"] * case["N"]
        # read x (and the residual), write y; a multiplication and a sum an element beside the generator
        return {"bytes": n * size[case["dtype"]] * (3 if case["residual"] else 2), "flops": 2 * n}
    if case["kind"] == "rope":
        rows = case["B"] * case["T"]
        n = rows * (case["HQ"] + case["HK"]) * case["D"]
        x, y = size[case["x"]], size[case["y"]]
        # the tables: a row of cosines and sines a position (shared by the batch where it is long)
        tables = (case["B"] if case["T"] == 1 else case["T"]) * case["R"] * 4
        moved = n * (x + y) if case["dir"] == "fwd" else n * (x + 2 * y)
        return {"bytes": moved + tables + 8 * case["D"] * (1 if case["dir"] == "fwd" else 2),
                "flops": (8 if case["dir"] == "fwd" else 16) * n}
    B, TQ, TK, HQ, HK, D = (case[c] for c in ("B", "TQ", "TK", "HQ", "HK", "D"))
    # ragged lengths are drawn from a quarter to all of the keys: 5/8 of them on average
    share = 0.625 if case["lens"] == "ragged" else 1.0
    keys = TK * share
    seen = TQ * (TK - TQ) + TQ * (TQ + 1) / 2 if case["causal"] else TQ * TK
    pairs = B * HQ * seen * share
    e = size[case["dtype"]]
    nq, nk = B * TQ * HQ * D * e, B * keys * HK * D * e
    if case["dir"] == "fwd":
        # q, k, v in, o and the log-sum-exp out; two products
        return {"bytes": 2 * nq + 2 * nk + 4 * B * HQ * TQ, "flops": 4 * D * pairs}
    # q, k, v, o, do, log-sum-exp in, dq, dk, dv out; five products (scores and dP anew, dv, dq, dk)
    return {"bytes": 4 * nq + 4 * nk + 4 * B * HQ * TQ, "flops": 10 * D * pairs}

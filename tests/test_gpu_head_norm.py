"""mt_qk_norm_rope_fwd and mt_qk_norm_rope_bwd against the formulas in 64 bits.

Bounds, with u = 2^-8 for a bf16 result (0 for fp32) and f = 1e-5 for the fp32
arithmetic (sums of at most 1024 squares and a few products, each with relative
error 2^-24): a rotated value is off by f of |a| + |b| of its pair and u of
itself; dx by f of r (|e| + |n| mean |n e|), where e of a rotated pair counts
with both its terms; dw by 1e-4 of its absolute terms, the project's bar for
fp32 sums.
"""
import math

import pytest
import torch

from attention_reference import check

pytestmark = pytest.mark.gpu

from paper_2602_00125_amd import binding as b  # noqa: E402  (a missing library fails the module)

DEV = "cuda:0"
DT = {"f32": torch.float32, "bf16": torch.bfloat16}
EPS = 1e-5
F = 1e-5


def draw(shape, dtype, seed):
    g = torch.Generator("cpu")
    g.manual_seed(seed)
    return torch.randn(shape, generator=g).to(DT[dtype]).to(DEV)


def tables(B, T, R, seed, shared=False):
    g = torch.Generator("cpu")
    g.manual_seed(seed)
    a = 6.3 * torch.rand((1 if shared else B, T, R // 2), generator=g)
    return [f(a).to(DEV).expand(B, T, R // 2) for f in (torch.cos, torch.sin)]


def pairs(x, R, inter):
    return (x[..., 0:R:2], x[..., 1:R:2]) if inter else (x[..., :R // 2], x[..., R // 2:R])


def join(p, q, rest, inter):
    head = torch.stack([p, q], -1).flatten(-2) if inter else torch.cat([p, q], -1)
    return torch.cat([head, rest], -1)


def turn(x, cos, sin, inter, back=False):
    if cos is None:
        return x, x.abs()
    R = 2 * cos.shape[-1]
    p, q = pairs(x, R, inter)
    c, s = cos.double()[:, :, None], sin.double()[:, :, None] * (-1 if back else 1)
    size = p.abs() + q.abs()
    return join(p * c - q * s, q * c + p * s, x[..., R:], inter), join(size, size, x[..., R:].abs(), inter)


def weight(w, D):
    return torch.ones(D, dtype=torch.float64, device=DEV) if w is None else w.double()


def fwd_reference(x, w, cos, sin, inter, u):
    x = x.double()
    r = (x.square().mean(-1, keepdim=True) + EPS).rsqrt()
    y, size = turn(x * r * weight(w, x.shape[-1]), cos, sin, inter)
    return y, F * size + u * y.abs() + 1e-30


def bwd_reference(x, w, cos, sin, dy, inter, u):
    x = x.double()
    r = (x.square().mean(-1, keepdim=True) + EPS).rsqrt()
    n = x * r
    g, gs = turn(dy.double(), cos, sin, inter, back=True)
    W = weight(w, x.shape[-1])
    dx = r * (g * W - n * (n * g * W).mean(-1, keepdim=True))
    size = r * (gs * W.abs() + n.abs() * (n * gs * W).abs().mean(-1, keepdim=True))
    return dx, F * size + u * dx.abs() + 1e-30, (g * n).sum((0, 1, 2)), 1e-4 * (gs * n.abs()).sum((0, 1, 2)) + 1e-6


def workspace(n):
    return torch.empty(n, dtype=torch.uint8, device=DEV) if n else None


def run_case(B, T, HQ, HK, D, R, x="f32", y="f32", inter=False, weights=True, shared=False, move=lambda t: t, seed=0):
    q, k = move(draw((B, T, HQ, D), x, seed)), move(draw((B, T, HK, D), x, seed + 1))
    dyq, dyk = move(draw((B, T, HQ, D), y, seed + 2)), move(draw((B, T, HK, D), y, seed + 3))
    wq, wk = (draw((D,), "f32", seed + 4 + i) if weights else None for i in range(2))
    cos, sin = tables(B, T, R, seed + 6, shared) if R else (None, None)
    u = 2.0 ** -8 if y == "bf16" else 0.0
    new = lambda t: move(torch.full(t.shape, math.nan, dtype=DT[y], device=DEV))
    yq, yk = new(q), new(k)
    b.qk_norm_rope_fwd(q, k, wq, wk, cos, sin, yq, yk, eps=EPS, interleaved=inter)
    for name, t, w, got in (("yq", q, wq, yq), ("yk", k, wk, yk)):
        check(name, got, *fwd_reference(t, w, cos, sin, inter, u))
    dq, dk = new(q), new(k)
    dwq, dwk = (torch.full((D,), math.nan, device=DEV) for _ in range(2))
    ws = workspace(b.qk_norm_rope_bwd_workspace(q, k, wq, wk, cos, sin, dyq, dyk, dq, dk, dwq, dwk))
    b.qk_norm_rope_bwd(q, k, wq, wk, cos, sin, dyq, dyk, dq, dk, dwq, dwk, eps=EPS, interleaved=inter, workspace=ws)
    for s, t, w, dy, dx, dw in (("q", q, wq, dyq, dq, dwq), ("k", k, wk, dyk, dk, dwk)):
        want, bound, wd, bd = bwd_reference(t, w, cos, sin, dy, inter, u)
        check("d" + s, dx, want, bound)
        check("dw" + s, dw, wd, bd)


TYPES = [("f32", "f32"), ("bf16", "bf16"), ("f32", "bf16"), ("bf16", "f32")]


@pytest.mark.parametrize("inter", [False, True])
@pytest.mark.parametrize("x,y", TYPES)
@pytest.mark.parametrize("size", [(1, 1, 1, 1, 64, 64), (2, 37, 5, 2, 128, 128), (3, 50, 4, 4, 96, 48),
                                  (1, 129, 3, 1, 80, 80), (2, 9, 2, 2, 256, 64), (2, 500, 32, 8, 128, 128),
                                  (64, 1, 8, 2, 32, 32)], ids=str)
def test_sizes(size, x, y, inter):
    run_case(*size, x=x, y=y, inter=inter)


@pytest.mark.parametrize("inter", [False, True])
@pytest.mark.parametrize("D,R", [(1, 0), (2, 2), (7, 4), (33, 30), (36, 12), (100, 100), (515, 130), (1024, 1024),
                                 (1000, 6)])
def test_widths(D, R, inter):
    run_case(2, 11, 3, 2, D, R, inter=inter)
    run_case(2, 11, 3, 2, D, R, x="bf16", y="bf16", inter=inter)


@pytest.mark.parametrize("weights", [False, True])
@pytest.mark.parametrize("R", [0, 64])
def test_without_weights_or_rotation(weights, R):
    run_case(2, 21, 4, 2, 64, R, weights=weights)
    run_case(2, 21, 4, 2, 64, R, x="bf16", y="bf16", weights=weights, shared=True)


@pytest.mark.parametrize("layout", ["heads_first", "odd_pitch", "offset"])
def test_layouts(layout):
    def move(t):
        if layout == "heads_first":
            return t.transpose(1, 2).contiguous().transpose(1, 2)
        if layout == "odd_pitch":
            buf = torch.zeros(*t.shape[:3], t.shape[3] + 1, dtype=t.dtype, device=DEV)
            buf[..., :-1] = t
            return buf[..., :-1]
        buf = torch.zeros(t.numel() + 1, dtype=t.dtype, device=DEV)
        buf[1:] = t.flatten()
        return buf[1:].view(t.shape)
    for x, y in TYPES:
        run_case(2, 30, 4, 2, 64, 64, x=x, y=y, move=move)


def test_packed_projection_and_gradient():
    """q and k are views of one projection and their gradients of one buffer: nothing else of it is written."""
    B, T, HQ, HK, D = 2, 19, 4, 2, 64
    qkv, dqkv = draw((B, T, (HQ + 2 * HK) * D), "f32", 0), torch.full((B, T, (HQ + 2 * HK) * D), 7.0, device=DEV)
    cut = lambda w: (w[..., :HQ * D].unflatten(-1, (HQ, D)), w[..., HQ * D:(HQ + HK) * D].unflatten(-1, (HK, D)))
    (q, k), (dq, dk) = cut(qkv), cut(dqkv)
    cos, sin = tables(B, T, D, 1)
    wq, wk, dyq, dyk = draw((D,), "f32", 2), draw((D,), "f32", 3), draw(q.shape, "f32", 4), draw(k.shape, "f32", 5)
    b.qk_norm_rope_bwd(q, k, wq, wk, cos, sin, dyq, dyk, dq, dk, eps=EPS)
    for t, w, dy, dx in ((q, wq, dyq, dq), (k, wk, dyk, dk)):
        want, bound, _, _ = bwd_reference(t, w, cos, sin, dy, False, 0.0)
        check("dx", dx, want, bound)
    assert (dqkv[..., (HQ + HK) * D:] == 7.0).all()


def test_queries_alone_accumulate_and_skipped_outputs():
    B, T, H, D = 2, 40, 4, 64
    q, dy, w = draw((B, T, H, D), "f32", 0), draw((B, T, H, D), "f32", 1), draw((D,), "f32", 2)
    cos, sin = tables(B, T, D, 3)
    want, bound, wd, bd = bwd_reference(q, w, cos, sin, dy, False, 0.0)
    ws = workspace(b.qk_norm_rope_bwd_workspace(q, None, w, None, cos, sin, dy, None, None, None, w.clone()))
    dw, dq = torch.full((D,), 3.0, device=DEV), draw(q.shape, "f32", 4)
    was = dq.clone()
    b.qk_norm_rope_bwd(q, None, w, None, cos, sin, dy, None, None, None, dw, eps=EPS, accumulate=True, workspace=ws)
    check("dw", dw, wd + 3.0, bd + 1e-6)
    b.qk_norm_rope_bwd(q, None, w, None, cos, sin, dy, None, dq, eps=EPS, accumulate=True)
    check("dq", dq, want + was.double(), bound + 1e-6 * (1 + was.double().abs()))


def test_zero_rows_and_empty_tensors():
    x = torch.zeros(2, 3, 2, 64, device=DEV)
    y = torch.full_like(x, math.nan)
    cos, sin = tables(2, 3, 64, 0)
    b.qk_norm_rope_fwd(x, None, None, None, cos, sin, y, None, eps=EPS)
    assert (y == 0).all()
    e = torch.zeros(0, 3, 2, 64, device=DEV)
    ce, se = tables(0, 3, 64, 0)
    b.qk_norm_rope_fwd(e, None, None, None, ce, se, e.clone(), None)
    dw = torch.full((64,), math.nan, device=DEV)
    ws = workspace(b.qk_norm_rope_bwd_workspace(e, None, None, None, ce, se, e, None, None, None, dw))
    b.qk_norm_rope_bwd(e, None, None, None, ce, se, e, None, None, None, dw, workspace=ws)
    assert (dw == 0).all()


def test_gradients_against_differences():
    """Central differences of the fp32 forward along random unit directions: truncation of order h^2, the
    forward's error (1e-6 a value, at random over the n values of dy) divided by 2 h."""
    B, T, H, D = 1, 12, 2, 64
    q, dy, w = draw((B, T, H, D), "f32", 0), draw((B, T, H, D), "f32", 1), draw((D,), "f32", 2)
    cos, sin = tables(B, T, D, 3)
    dq, dw = torch.empty_like(q), torch.empty_like(w)
    ws = workspace(b.qk_norm_rope_bwd_workspace(q, None, w, None, cos, sin, dy, None, dq, None, dw))
    b.qk_norm_rope_bwd(q, None, w, None, cos, sin, dy, None, dq, None, dw, eps=EPS, workspace=ws)
    h = 1e-2
    for i, (t, g) in enumerate(((q, dq), (w, dw))):
        way = draw(t.shape, "f32", 9 + i)
        way /= way.norm()

        def loss(sign):
            y = torch.empty_like(q)
            x, v = (a + sign * h * way if a is t else a for a in (q, w))
            b.qk_norm_rope_fwd(x, None, v, None, cos, sin, y, None, eps=EPS)
            return (y.double() * dy.double()).sum().item()

        slope, want = (loss(1) - loss(-1)) / (2 * h), (g.double() * way.double()).sum().item()
        assert abs(slope - want) <= 1e-6 * math.sqrt(dy.numel()) / (2 * h) + 10 * h * h


def test_same_bits_every_time():
    q, dy, w = draw((4, 700, 8, 128), "bf16", 0), draw((4, 700, 8, 128), "bf16", 1), draw((128,), "f32", 2)
    cos, sin = tables(4, 700, 128, 3)
    outs = []
    for _ in range(2):
        dq, dw = torch.empty_like(q), torch.empty_like(w)
        ws = workspace(b.qk_norm_rope_bwd_workspace(q, None, w, None, cos, sin, dy, None, dq, None, dw))
        b.qk_norm_rope_bwd(q, None, w, None, cos, sin, dy, None, dq, None, dw, workspace=ws)
        outs.append((dq, dw))
    assert torch.equal(outs[0][0], outs[1][0]) and torch.equal(outs[0][1], outs[1][1])


def test_more_rows_than_threads_along_a_grid():
    T = (1 << 26) + 5  # a wave a row: 2^32 threads and some
    x = torch.empty((1, T, 1, 1), dtype=torch.bfloat16, device=DEV).fill_(3.0)
    y = torch.full_like(x, math.nan)
    b.qk_norm_rope_fwd(x, None, None, None, None, None, y, None, eps=0.0)
    torch.cuda.synchronize()
    assert (y == 1).all()

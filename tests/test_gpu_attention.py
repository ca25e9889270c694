"""mt_attention_fwd and mt_attention_bwd against plain attention in 64 bits."""
import math

import pytest
import torch

from attention_reference import check, reference

pytestmark = pytest.mark.gpu

from paper_2602_00125_amd import binding as b  # noqa: E402  (a missing library fails the module)

DEV = "cuda:0"
DT = {"f32": torch.float32, "bf16": torch.bfloat16}


def draw(shape, dtype, seed):
    g = torch.Generator("cpu")
    g.manual_seed(seed)
    return torch.randn(shape, generator=g).to(DT[dtype]).to(DEV)


def nan_like(shape, dtype):
    return torch.full(shape, math.nan, dtype=DT[dtype] if isinstance(dtype, str) else dtype, device=DEV)


def workspace(n):
    return torch.empty(n, dtype=torch.uint8, device=DEV) if n else None


def forward(q, k, v, o=None, use_ws=True, **kw):
    B, TQ, HQ, _ = q.shape
    o = nan_like(q.shape, q.dtype) if o is None else o
    lse = nan_like((B, HQ, TQ), "f32")
    qkw = {n: kw[n] for n in kw if n != "scale"}
    ws = workspace(b.attention_fwd_workspace(q, k, v, o, lse, **qkw)) if use_ws else None
    b.attention_fwd(q, k, v, o, lse, workspace=ws, **kw)
    return o, lse


def backward(q, k, v, o, lse, dout, outs=None, accumulate=False, **kw):
    dq, dk, dv = outs or (nan_like(q.shape, q.dtype), nan_like(k.shape, q.dtype), nan_like(k.shape, q.dtype))
    qkw = {n: kw[n] for n in kw if n != "scale"}
    ws = workspace(b.attention_bwd_workspace(q, k, v, o, lse, dout, dq, dk, dv, **qkw))
    b.attention_bwd(q, k, v, o, lse, dout, dq, dk, dv, accumulate=accumulate, workspace=ws, **kw)
    return dq, dk, dv


def run_case(dtype, B, TQ, TK, HQ, HK, D, causal=False, lens=None, start=None, seed=0, scale=None, use_ws=True):
    q, k, v = (draw((B, t, h, D), dtype, seed + i) for i, (t, h) in enumerate(((TQ, HQ), (TK, HK), (TK, HK))))
    dout = draw((B, TQ, HQ, D), dtype, seed + 3)
    kv_len = None if lens is None else torch.tensor(lens, dtype=torch.int32, device=DEV)
    q_start = None if start is None else torch.tensor(start, dtype=torch.int32, device=DEV)
    kw = dict(causal=causal, kv_len=kv_len, q_start=q_start)
    o, lse = forward(q, k, v, scale=scale, use_ws=use_ws, **kw)
    grads = backward(q, k, v, o, lse, dout, scale=scale, **kw)
    torch.cuda.synchronize()
    ref = reference(q, k, v, D ** -0.5 if scale is None else scale, dout=dout, **kw)
    for name, got in zip(("o", "lse", "dq", "dk", "dv"), (o, lse, *grads)):
        check(name, got, *ref[name])


@pytest.fixture
def splits():
    """Sets how the forward shares out the keys (see mt_debug_set) for one test."""
    yield lambda n: b.debug_set("attn_splits", n)
    b.debug_set("attn_splits", -1)


# lengths around the tiles of 32, 64 and 128 tokens; every head width class; grouped heads
SIZES = [(1, 1, 1, 1, 1, 8), (2, 1, 5, 4, 2, 64), (1, 33, 31, 3, 1, 32), (2, 64, 64, 2, 2, 64), (1, 65, 129, 4, 4, 128),
         (2, 127, 200, 6, 2, 96), (1, 128, 128, 8, 1, 80), (1, 257, 383, 2, 1, 112), (1, 509, 383, 4, 2, 128),
         (3, 96, 160, 2, 1, 16), (1, 700, 700, 1, 1, 128)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("size", SIZES, ids=str)
def test_sizes(dtype, causal, size):
    run_case(dtype, *size, causal=causal)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n", [0, 1, 3, 64])
def test_forward_by_blocks_and_by_shares_of_the_keys(dtype, n, splits):
    """Every size by blocks of 128 queries, by one share and by shares of a few tiles or none, ragged too."""
    splits(n)
    for size in SIZES:
        for causal in (False, True):
            B, TQ, TK, HQ, HK, D = size
            lens = None if causal else [max(0, TK - 40 * i) for i in range(B)]
            run_case(dtype, *size, causal=causal, lens=lens)
    run_case(dtype, 2, 20, 90, 4, 2, 33, causal=True)
    run_case(dtype, 2, 50, 50, 4, 2, 64, causal=True, lens=[0, 33])
    run_case(dtype, 1, 8, 2000, 4, 1, 128, causal=True, lens=[1500], use_ws=False)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("D", [64, 96, 128, 50])
def test_more_blocks_than_compute_units(dtype, D, splits):
    """Grids of more than 256 blocks of 128 queries (or keys), where fewer waves share those of a block."""
    splits(0)
    run_case(dtype, 5, 260, 200, 20, 4, D, causal=True, lens=[200, 0, 77, 130, 199])
    run_case(dtype, 4, 290, 290, 24, 8, D, causal=True)
    run_case(dtype, 5, 150, 300, 20, 20, D, causal=True, lens=[300, 300, 0, 1, 170])
    run_case(dtype, 5, 260, 200, 20, 4, D, lens=[200, 0, 77, 130, 199])
    run_case(dtype, 7, 300, 300, 28, 7, D, causal=True)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_one_token_against_long_caches(dtype):
    """Single tokens and short chunks at the ends of ragged caches, given as views of a longer buffer."""
    B, TK, HQ, HK, D = 3, 5000, 8, 2, 128
    k, v = (draw((B, TK + 100, HK, D), dtype, i)[:, :TK] for i in range(2))
    lens = torch.tensor([5000, 1, 2777], dtype=torch.int32, device=DEV)
    for TQ in (1, 3):
        q = draw((B, TQ, HQ, D), dtype, 7 + TQ)
        kw = dict(causal=True, kv_len=lens, q_start=(lens - TQ).int())
        ref = reference(q, k, v, D ** -0.5, **kw)
        for name, got in zip(("o", "lse"), forward(q, k, v, **kw)):
            check(name, got, *ref[name])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("D", [1, 3, 20, 33, 65, 100, 127])
def test_head_widths_without_vectors(dtype, D):
    run_case(dtype, 2, 70, 67, 4, 2, D, causal=True)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("TQ,TK", [(150, 150), (1, 300), (40, 300), (300, 40)])
def test_ragged_lengths(dtype, causal, TQ, TK):
    """Lengths of nothing, one, a tile's edge and all; negative and too long ones are clamped. With more
    queries than keys the first causal queries see nothing."""
    lens = [0, 1, min(64, TK), TK, -3, TK + 7, TK // 2]
    run_case(dtype, len(lens), TQ, TK, 4, 2, 64, causal=causal, lens=lens)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_query_positions(dtype):
    """Chunks of queries at their own positions: before every key, inside, past the end, far out of range."""
    start = [-200, -5, 0, 17, 100, 1000, 2 ** 31 - 1, -2 ** 31]
    run_case(dtype, len(start), 70, 130, 2, 1, 64, causal=True, start=start, lens=[130, 130, 1, 60, 130, 99, 64, 130])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("D", [64, 128, 50])
def test_garbage_past_the_length_is_not_used(dtype, D):
    B, TQ, TK, H = 3, 45, 150, 2
    q, k, v, dout = (draw((B, t, H, D), dtype, i) for i, t in enumerate((TQ, TK, TK, TQ)))
    kv_len = torch.tensor([70, 0, 129], dtype=torch.int32, device=DEV)
    for i, n in enumerate(kv_len.tolist()):
        k[i, n:], v[i, n:] = math.nan, math.inf
    for causal in (False, True):
        o, lse = forward(q, k, v, causal=causal, kv_len=kv_len)
        grads = backward(q, k, v, o, lse, dout, causal=causal, kv_len=kv_len)
        ref = reference(q, k, v, D ** -0.5, causal=causal, kv_len=kv_len, dout=dout)
        for name, got in zip(("o", "lse", "dq", "dk", "dv"), (o, lse, *grads)):
            check(name, got, *ref[name])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_garbage_keys_past_the_causal_edge_do_not_change_scores(dtype):
    """A key that no query of the call sees (a cache's stale end) may hold anything."""
    q, k, v = (draw((1, t, 2, 64), dtype, i) for i, t in enumerate((10, 300, 300)))
    start = torch.tensor([90], dtype=torch.int32, device=DEV)  # queries at 90 .. 99
    want = forward(q, k, v, causal=True, q_start=start)
    k[:, 128:], v[:, 128:] = math.nan, math.nan
    got = forward(q, k, v, causal=True, q_start=start)
    for x, y in zip(got, want):
        assert torch.equal(x, y)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shift", [-60.0, 60.0])
def test_large_scores(dtype, shift):
    """Scores far from zero, growing and falling along the keys: the running maximum moves."""
    B, T, H, D = 1, 300, 2, 64
    q, k, v, dout = (draw((B, T, H, D), dtype, i) for i in range(4))
    ramp = torch.linspace(0, abs(shift), T, device=DEV)
    ramp = ramp if shift > 0 else ramp.flip(0)
    q[..., 0], k[..., 0] = 8.0, ramp[None, :, None].to(q.dtype)
    for causal in (False, True):
        o, lse = forward(q, k, v, causal=causal)
        grads = backward(q, k, v, o, lse, dout, causal=causal)
        ref = reference(q, k, v, D ** -0.5, causal=causal, dout=dout)
        for name, got in zip(("o", "lse", "dq", "dk", "dv"), (o, lse, *grads)):
            check(name, got, *ref[name])


@pytest.mark.parametrize("scale", [1e-3, 0.7])
def test_scale(scale):
    run_case("f32", 1, 90, 110, 2, 2, 32, scale=scale)
    run_case("bf16", 1, 90, 110, 2, 2, 32, scale=scale)


def packed(B, T, HQ, HK, D, dtype, seed):
    w = draw((B, T, (HQ + 2 * HK) * D), dtype, seed)
    return w, [w[..., a * D:(a + h) * D].unflatten(-1, (h, D)) for a, h in ((0, HQ), (HQ, HK), (HQ + HK, HK))]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("layout", ["packed", "heads_first", "odd_pitch", "offset"])
def test_layouts(dtype, layout):
    """Packed projections (gradients into one packed buffer too), [B, H, T, D] memory, pitches and bases that do
    not allow vectors."""
    B, T, HQ, HK, D = 2, 77, 4, 2, 64
    w, (q, k, v) = packed(B, T, HQ, HK, D, dtype, 1)
    dout = draw((B, T, HQ, D), dtype, 2)
    outs = None
    if layout == "packed":
        _, outs = packed(B, T, HQ, HK, D, dtype, 3)
    else:
        def move(x):
            x = x.contiguous()
            if layout == "heads_first":
                return x.transpose(1, 2).contiguous().transpose(1, 2)
            if layout == "odd_pitch":
                buf = torch.zeros(*x.shape[:3], D + 3, dtype=x.dtype, device=DEV)
                buf[..., :D] = x
                return buf[..., :D]
            buf = torch.zeros(x.numel() + 1, dtype=x.dtype, device=DEV)
            buf[1:] = x.flatten()
            return buf[1:].view(x.shape)
        q, k, v, dout = (move(x) for x in (q, k, v, dout))
    o, lse = forward(q, k, v, causal=True)
    grads = backward(q, k, v, o, lse, dout, outs=outs, causal=True)
    ref = reference(q, k, v, D ** -0.5, causal=True, dout=dout)
    for name, got in zip(("o", "lse", "dq", "dk", "dv"), (o, lse, *grads)):
        check(name, got, *ref[name])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_accumulate_and_skipped_outputs(dtype):
    B, T, HQ, HK, D = 2, 100, 4, 2, 64
    q, k, v, dout = (draw((B, T, h, D), dtype, i) for i, h in enumerate((HQ, HK, HK, HQ)))
    kv_len = torch.tensor([100, 37], dtype=torch.int32, device=DEV)
    o, lse = forward(q, k, v, causal=True, kv_len=kv_len)
    full = backward(q, k, v, o, lse, dout, causal=True, kv_len=kv_len)
    for keep in range(1, 8):
        outs = [torch.full_like(t, math.nan) if keep >> i & 1 else None for i, t in enumerate(full)]
        backward(q, k, v, o, lse, dout, outs=outs, causal=True, kv_len=kv_len)
        for got, want in zip(outs, full):
            assert got is None or torch.equal(got, want)
    base = [draw(t.shape, dtype, 9 + i) for i, t in enumerate(full)]
    outs = [t.clone() for t in base]
    backward(q, k, v, o, lse, dout, outs=outs, accumulate=True, causal=True, kv_len=kv_len)
    ref = reference(q, k, v, D ** -0.5, causal=True, kv_len=kv_len, dout=dout)
    u = 2.0 ** -8 if dtype == "bf16" else 2.0 ** -24
    for name, got, was in zip(("dq", "dk", "dv"), outs, base):
        want, bound = ref[name]
        want = want + was.double()
        check(name, got, want, bound + 1.05 * u * want.abs())


def test_empty_tensors():
    for B, TQ, TK, HQ, HK in ((0, 3, 3, 2, 1), (2, 0, 3, 2, 1), (2, 3, 0, 2, 1), (1, 3, 3, 0, 2)):
        q, k, v, dout = (draw((B, t, h, 64), "bf16", 0) for t, h in ((TQ, HQ), (TK, HK), (TK, HK), (TQ, HQ)))
        o, lse = forward(q, k, v)
        assert (o == 0).all() and (lse == -math.inf).all() if TK == 0 else True
        dq, dk, dv = backward(q, k, v, o, lse, dout)
        if TQ == 0 or TK == 0:
            for t in (dq, dk, dv):
                assert (t == 0).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_same_bits_every_time_and_on_another_stream(dtype):
    B, T, HQ, HK, D = 2, 300, 8, 2, 128
    q, k, v, dout = (draw((B, T, h, D), dtype, i) for i, h in enumerate((HQ, HK, HK, HQ)))
    o, lse = forward(q, k, v, causal=True)
    want = [o, lse, *backward(q, k, v, o, lse, dout, causal=True)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        o2, lse2 = forward(q, k, v, causal=True)
        got = [o2, lse2, *backward(q, k, v, o2, lse2, dout, causal=True)]
    torch.cuda.current_stream().wait_stream(side)
    for x, y in zip(got, want):
        assert torch.equal(x, y)


@pytest.mark.parametrize("causal", [False, True])
def test_gradients_against_differences(causal):
    """<dout, o> along random directions: central differences of the fp32 forward, summed in 64 bits. With step h
    the truncation is h^2 / 6 times a third derivative of order 1 a direction, and the forward's error (about
    1e-6 a value over n values of dout, adding up at random) is divided by 2 h."""
    B, T, H, D = 1, 40, 2, 32
    q, k, v, dout = (draw((B, T, H, D), "f32", i) for i in range(4))
    o, lse = forward(q, k, v, causal=causal)
    grads = backward(q, k, v, o, lse, dout, causal=causal)
    h = 1e-2
    for i, (t, g) in enumerate(zip((q, k, v), grads)):
        way = draw(t.shape, "f32", 50 + i)
        way /= way.norm()

        def loss(sign):
            args = [x + sign * h * way if x is t else x for x in (q, k, v)]
            return (forward(*args, causal=causal)[0].double() * dout.double()).sum().item()

        slope = (loss(1) - loss(-1)) / (2 * h)
        want = (g.double() * way.double()).sum().item()
        assert abs(slope - want) <= 1e-6 * math.sqrt(dout.numel()) / (2 * h) + 10 * h * h, (i, slope, want)


def test_replays_from_a_graph():
    B, T, HQ, HK, D = 2, 200, 4, 2, 64
    q, k, v, dout = (draw((B, T, h, D), "bf16", i) for i, h in enumerate((HQ, HK, HK, HQ)))
    lens = torch.tensor([150, 200], dtype=torch.int32, device=DEV)
    o, lse = torch.empty_like(q), torch.empty(B, HQ, T, device=DEV)
    grads = [torch.empty_like(t) for t in (q, k, v)]
    wf = workspace(b.attention_fwd_workspace(q, k, v, o, lse, kv_len=lens, causal=True))
    wb = workspace(b.attention_bwd_workspace(q, k, v, o, lse, dout, *grads, kv_len=lens, causal=True))

    def step():
        b.attention_fwd(q, k, v, o, lse, kv_len=lens, causal=True, workspace=wf)
        b.attention_bwd(q, k, v, o, lse, dout, *grads, kv_len=lens, causal=True, workspace=wb)

    step()
    torch.cuda.synchronize()
    eager = [t.clone() for t in (o, lse, *grads)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step()
    for _ in range(3):
        for t in (o, lse, *grads):
            t.fill_(math.nan)
        g.replay()
        torch.cuda.synchronize()
        for got, want in zip((o, lse, *grads), eager):
            assert torch.equal(got, want)
        step()
        torch.cuda.synchronize()
        for got, want in zip((o, lse, *grads), eager):
            assert torch.equal(got, want)


# pitch of a token's row in elements: vectors at the longest pitch that they serve, and
# by element past it; 1300 rows reach past 2^31 elements and 2^32 bytes
@pytest.mark.parametrize("dtype,pitch", [("bf16", 1 << 21), ("bf16", (1 << 21) + 3), ("f32", 1 << 20), ("f32", (1 << 21) + 8)])
def test_offsets_past_32_bits(dtype, pitch):
    T, H, D = 1300, 2, 32
    W = H * D
    x = torch.empty(T * pitch, dtype=DT[dtype], device=DEV)
    assert x.numel() * x.element_size() > 1 << 32
    q, k, v, o, dout, dq, dk, dv = (x.as_strided((1, T, H, D), (T * pitch, pitch, D, 1), W * i) for i in range(8))
    close = [draw((1, T, H, D), dtype, i) for i in range(4)]
    for far, near in zip((q, k, v, dout), close):
        far.copy_(near)
    want_o, want_lse = forward(*close[:3], causal=True)
    want = backward(*close[:3], want_o, want_lse, close[3], causal=True)
    _, lse = forward(q, k, v, o, causal=True)
    backward(q, k, v, o, lse, dout, (dq, dk, dv), causal=True)
    few, few_lse = forward(q[:, -3:], k, v, causal=True)  # the last tokens against a long cache
    torch.cuda.synchronize()
    assert torch.equal(lse, want_lse) and torch.equal(o, want_o)
    for got, near in zip((dq, dk, dv), want):
        assert torch.equal(got, near)
    ref = reference(close[0][:, -3:], *close[1:3], D ** -0.5, causal=True)
    check("o", few, *ref["o"])
    check("lse", few_lse, *ref["lse"])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("case", [(1, 71, 71, 8, 1, 96), (1, 600, 600, 8, 1, 128), (2, 257, 190, 6, 2, 50), (1, 1100, 40, 3, 1, 64)])
def test_gradients_of_few_key_blocks(dtype, case):
    """Blocks of keys fewer than the compute units: the query tiles are shared out, some shares without a tile."""
    B, TK = case[0], case[2]
    run_case(dtype, *case, causal=True)
    run_case(dtype, *case, lens=[TK // 3] * B)
    run_case(dtype, *case, causal=True, start=[TK - 5] * B)

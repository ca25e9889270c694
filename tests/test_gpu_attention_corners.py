"""Corners of attention and the head norms."""
import math

import pytest
import torch

from attention_reference import check, reference

pytestmark = pytest.mark.gpu

from paper_2602_00125_amd import binding as b  # noqa: E402  (a missing library fails the module)
from test_gpu_attention import DEV, backward, draw, forward, splits  # noqa: E402,F401


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("B,TQ,TK,HK,D", [(1, 3, 3, 2, 64), (2, 40, 300, 3, 128), (9, 130, 77, 8, 50)])
def test_keys_without_query_heads_have_no_gradient(dtype, causal, B, TQ, TK, HK, D):
    """dk and dv are sums over no query head: zero, and left as they were where they accumulate."""
    q, k, v, dout = (draw((B, t, h, D), dtype, i) for i, (t, h) in enumerate(((TQ, 0), (TK, HK), (TK, HK), (TQ, 0))))
    lens = torch.full((B,), TK // 2, dtype=torch.int32, device=DEV)
    for kv_len in (None, lens):
        o, lse = forward(q, k, v, causal=causal, kv_len=kv_len)
        dq, dk, dv = backward(q, k, v, o, lse, dout, causal=causal, kv_len=kv_len)
        assert (dk == 0).all() and (dv == 0).all()
        was = [draw(k.shape, dtype, 7), draw(k.shape, dtype, 8)]
        outs = (dq, *(t.clone() for t in was))
        backward(q, k, v, o, lse, dout, outs=outs, accumulate=True, causal=causal, kv_len=kv_len)
        assert torch.equal(outs[1], was[0]) and torch.equal(outs[2], was[1])


@pytest.mark.parametrize("D", [64, 50])  # by vectors and by element
@pytest.mark.parametrize("none", ["q", "k"])
def test_norm_gradients_with_no_heads_on_one_side(D, none):
    """Queries or keys of no heads, whose empty tensors have no memory: the others' gradient is what it is alone."""
    B, T, H = 2, 21, 3
    x, dy, w = draw((B, T, H, D), "f32", 0), draw((B, T, H, D), "f32", 1), draw((D,), "f32", 2)
    a = 6.3 * torch.rand((B, T, D // 2), generator=torch.Generator("cpu").manual_seed(3))
    cos, sin = a.cos().to(DEV), a.sin().to(DEV)
    want = torch.empty_like(x)
    b.qk_norm_rope_bwd(x, None, w, None, cos, sin, dy, None, want)
    empty = torch.empty(B, T, 0, D, device=DEV)
    assert empty.data_ptr() == 0
    dx = torch.full_like(x, math.nan)
    ins, outs = [(empty, empty), (x, dy)], [empty, dx]
    (q, dyq), (k, dyk) = ins if none == "q" else ins[::-1]
    dq, dk = outs if none == "q" else outs[::-1]
    b.qk_norm_rope_bwd(q, k, w, w, cos, sin, dyq, dyk, dq, dk)
    assert torch.equal(dx, want)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n", [100, -100])
def test_the_ends_of_the_range_of_scales(dtype, n):
    """A scale of 2^-100 (2^100) with queries and keys of as much larger (smaller) values: powers of two change no
    rounding, so o, lse and dv are the bits of scale 1/8, dq and dk those times the powers."""
    B, T, HQ, HK, D = 2, 200, 4, 2, 64
    q, k, v, dout = (draw((B, T, h, D), dtype, i) for i, h in enumerate((HQ, HK, HK, HQ)))
    fq, fk = 2.0 ** (n // 2 - 2), 2.0 ** (n // 2 - 1)  # 2^-100 fq fk = 1 / 8
    outs = []
    for x, y, scale in ((q, k, 0.125), (q * fq, k * fk, 2.0 ** -n)):
        o, lse = forward(x, y, v, scale=scale, causal=True)
        outs.append([o, lse, *backward(x, y, v, o, lse, dout, scale=scale, causal=True)])
    (o, lse, dq, dk, dv), (o2, lse2, dq2, dk2, dv2) = outs
    assert torch.equal(o2, o) and torch.equal(lse2, lse) and torch.equal(dv2, dv)
    assert torch.equal(dq2 * fq, dq) and torch.equal(dk2 * fk, dk)


@pytest.mark.parametrize("n", [-1, 3])
def test_more_rows_than_a_launch_of_a_block_a_row_has(n, splits):
    """32 heads of 2^20 queries: 2^25 rows, which only the join of shared-out keys could not take."""
    splits(n)
    TQ, TK, HQ, D = 1 << 20, 64, 32, 8
    q, dout = (torch.randn((1, TQ, HQ, D), generator=torch.Generator(DEV).manual_seed(i), device=DEV).bfloat16() for i in range(2))
    k, v = draw((1, TK, 1, D), "bf16", 2), draw((1, TK, 1, D), "bf16", 3)
    o, lse = forward(q, k, v)
    dq, dk, dv = backward(q, k, v, o, lse, dout)
    sums = {"dk": [0.0, 0.0], "dv": [0.0, 0.0]}
    step = 1 << 16
    for t in range(0, TQ, step):
        cut = slice(t, t + step)
        ref = reference(q[:, cut], k, v, D ** -0.5, dout=dout[:, cut])
        for name, got in (("o", o[:, cut]), ("lse", lse[:, :, cut]), ("dq", dq[:, cut])):
            check(name, got, *ref[name])
        for name, s in sums.items():
            s[0], s[1] = s[0] + ref[name][0], s[1] + ref[name][1]
    for name, got in (("dk", dk), ("dv", dv)):
        check(name, got, *sums[name])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_heads_of_a_packed_buffer_side_by_side(dtype):
    """Each head's query, key and value next to one another ([B, T, H, 3, D]), the gradients laid out the same."""
    B, T, H, D = 2, 77, 3, 64
    qkv, dout = draw((B, T, H, 3, D), dtype, 0), draw((B, T, H, D), dtype, 1)
    grads = torch.full_like(qkv, math.nan)
    q, k, v = qkv.unbind(3)
    o, lse = forward(q, k, v, causal=True)
    backward(q, k, v, o, lse, dout, outs=grads.unbind(3), causal=True)
    ref = reference(q, k, v, D ** -0.5, causal=True, dout=dout)
    for name, got in zip(("o", "lse", "dq", "dk", "dv"), (o, lse, *grads.unbind(3))):
        check(name, got, *ref[name])

"""Host-side validation of attention, the head norms with rotation and dropout: every bad argument is reported with
the documented status before any HIP call. No case here passes validation, so nothing is ever launched and no GPU is
needed."""
import ctypes
import math

import pytest
import torch

from helpers import load_binding

b = load_binding()

from test_abi_host import BF16, D, F32, R  # noqa: E402

I32 = b.I32
B, TQ, TK, HQ, HK, W = 2, 6, 10, 4, 2, 16


def heads(t, h, ptr, dtype=F32, stride=None, batch=B, width=W):
    return D([batch, t, h, width], dtype, ptr, stride)


def args(**kw):
    """q, k, v, kv_len, q_start, o, lse and the gradients of a valid call, some replaced."""
    a = dict(q=heads(TQ, HQ, 0x100000), k=heads(TK, HK, 0x200000), v=heads(TK, HK, 0x300000), kv_len=None, q_start=None,
             o=heads(TQ, HQ, 0x400000), lse=D([B, HQ, TQ], ptr=0x500000), dout=heads(TQ, HQ, 0x600000),
             dq=heads(TQ, HQ, 0x700000), dk=heads(TK, HK, 0x800000), dv=heads(TK, HK, 0x900000), scale=0.25, flags=0,
             ws=0x1000000, ws_bytes=B * HQ * TQ * 4)
    a.update(kw)
    return a


def fwd(**kw):
    a = args(**kw)
    return b.lib.mt_attention_fwd(*[R(a[n]) for n in ("q", "k", "v", "kv_len", "q_start", "o", "lse")], a["scale"],
                                  a["flags"], None, 0, None)


def bwd(**kw):
    a = args(**kw)
    return b.lib.mt_attention_bwd(*[R(a[n]) for n in ("q", "k", "v", "kv_len", "q_start", "o", "lse", "dout", "dq", "dk",
                                                     "dv")], a["scale"], a["flags"], a["ws"], a["ws_bytes"], None)


NULL, NDIM, SHAPE, DTYPE, LAYOUT, ALIAS, WS, INVALID = 1, 2, 3, 4, 5, 6, 7, 9


@pytest.mark.parametrize("call", [fwd, bwd])
def test_attention_inputs(call):
    assert call(q=None) == NULL and call(k=None) == NULL and call(v=None) == NULL and call(o=None) == NULL
    assert call(q=D([B, TQ, HQ * W], ptr=0x100000)) == NDIM
    assert call(q=heads(TQ, HQ, 0)) == NULL
    assert call(k=heads(TK, HK, 0x200000, BF16)) == DTYPE
    assert call(q=heads(TQ, HQ, 0x100000, I32)) == DTYPE
    assert call(o=heads(TQ, HQ, 0x400000, BF16)) == DTYPE
    assert call(k=heads(TK, 3, 0x200000), v=heads(TK, 3, 0x300000)) == SHAPE    # 4 heads over 3
    assert call(k=heads(TK, 0, 0x200000), v=heads(TK, 0, 0x300000)) == SHAPE    # 4 heads over none
    assert call(v=heads(TK + 1, HK, 0x300000)) == SHAPE
    assert call(k=heads(TK, HK, 0x200000, batch=3), v=heads(TK, HK, 0x300000, batch=3)) == SHAPE
    assert call(k=heads(TK, HK, 0x200000, width=8), v=heads(TK, HK, 0x300000, width=8)) == SHAPE
    wide = {n: heads(t, h, p, width=129) for n, t, h, p in (("q", TQ, HQ, 0x100000), ("k", TK, HK, 0x200000),
                                                            ("v", TK, HK, 0x300000), ("o", TQ, HQ, 0x400000))}
    assert call(**wide) == SHAPE
    assert call(q=heads(TQ, HQ, 0x100000, stride=[TQ * HQ * W, HQ * W, 1, HQ])) == LAYOUT  # vectors not contiguous
    assert call(q=heads(TQ, HQ, 0x100000, stride=[-1, HQ * W, W, 1])) == LAYOUT
    for bad in (0.0, -1.0, math.inf, math.nan):
        assert call(scale=bad) == INVALID
    assert call(flags=2) == INVALID and call(flags=64) == INVALID
    assert call(lse=D([B, TQ, HQ], ptr=0x500000)) == SHAPE
    assert call(lse=D([B, HQ, TQ], BF16, 0x500000)) == DTYPE
    assert call(lse=D([B, HQ, TQ], ptr=0x500000, stride=[HQ * TQ, 1, HQ])) == LAYOUT
    for name in ("kv_len", "q_start"):
        assert call(**{name: D([B], F32, 0xa00000)}) == DTYPE
        assert call(**{name: D([B + 1], I32, 0xa00000)}) == SHAPE
        assert call(**{name: D([B, 1], I32, 0xa00000)}) == NDIM
        assert call(**{name: D([B], I32, 0)}) == NULL
        assert call(**{name: D([B], I32, 0xa00000, [2])}) == LAYOUT


def test_attention_outputs():
    assert fwd(flags=1) == INVALID                                       # the forward does not accumulate
    assert fwd(o=heads(TQ + 1, HQ, 0x400000)) == SHAPE
    assert fwd(o=heads(TQ, HQ, 0x400000, stride=[0, HQ * W, W, 1])) == LAYOUT   # written twice
    assert fwd(o=heads(TQ, HQ, 0x400000, stride=[TQ * HQ * W, W, W, 1])) == LAYOUT
    assert fwd(o=heads(TQ, HQ, 0x100000)) == ALIAS
    assert fwd(lse=D([B, HQ, TQ], ptr=0x400000)) == ALIAS
    assert fwd(kv_len=D([B], I32, 0x400004)) == ALIAS
    assert bwd(lse=None) == NULL and bwd(dout=None) == NULL and bwd(dq=None, dk=None, dv=None) == NULL
    assert bwd(dout=heads(TQ, HK, 0x600000)) == SHAPE
    assert bwd(dout=heads(TQ, HQ, 0x600000, BF16)) == DTYPE
    assert bwd(dq=heads(TK, HQ, 0x700000)) == SHAPE and bwd(dk=heads(TQ, HK, 0x800000)) == SHAPE
    assert bwd(dv=heads(TK, HK, 0x900000, BF16)) == DTYPE
    assert bwd(dv=heads(TK, HK, 0x800000)) == ALIAS and bwd(dq=heads(TQ, HQ, 0x600000)) == ALIAS
    assert bwd(dk=heads(TK, HK, 0x800000), q_start=D([B], I32, 0x800010)) == ALIAS
    assert bwd(ws=None, ws_bytes=0) == WS and bwd(ws_bytes=8) == WS and bwd(ws=0x1000004) == WS


def test_packed_views_are_apart():
    """Views of one packed buffer pass the overlap check (the next check refuses the call); views that share a
    column do not."""
    P = (HQ + 2 * HK) * W
    part = lambda h, col: D([B, TQ, h, W], F32, 0x700000 + 4 * col, [TQ * P, P, W, 1])
    call = lambda dq, dk, dv: bwd(k=heads(TQ, HK, 0x200000), v=heads(TQ, HK, 0x300000), dq=dq, dk=dk, dv=dv, ws=None)
    assert call(part(HQ, 0), part(HK, HQ * W), part(HK, (HQ + HK) * W)) == WS
    assert call(part(HQ, 0), part(HK, HQ * W - 1), part(HK, (HQ + HK) * W)) == ALIAS
    assert call(part(HQ, 0), part(HK, HQ * W), part(HK, (HQ + HK) * W + 1)) == ALIAS   # runs into the next token


def test_attention_workspace_queries():
    a = args()
    n = ctypes.c_size_t(1)
    names = ("q", "k", "v", "kv_len", "q_start", "o", "lse", "dout", "dq", "dk", "dv")
    assert b.lib.mt_attention_bwd_workspace(*[R(a[x]) for x in names], 0, ctypes.byref(n)) == 0
    assert n.value >= B * HQ * TQ * 4
    assert b.lib.mt_attention_fwd_workspace(*[R(a[x]) for x in names[:7]], 0, ctypes.byref(n)) == 0
    assert b.lib.mt_attention_bwd_workspace(*[R(a[x]) for x in names], 0, None) == NULL
    assert b.lib.mt_attention_fwd_workspace(*[R(a[x]) for x in names[:7]], 2, ctypes.byref(n)) == INVALID


def norm_args(**kw):
    a = dict(q=heads(TQ, HQ, 0x100000), k=heads(TQ, HK, 0x200000), wq=D([W], ptr=0x300000), wk=D([W], ptr=0x310000),
             cos=D([B, TQ, W // 2], ptr=0x400000), sin=D([B, TQ, W // 2], ptr=0x500000), yq=heads(TQ, HQ, 0x600000),
             yk=heads(TQ, HK, 0x700000), dq=heads(TQ, HQ, 0x800000), dk=heads(TQ, HK, 0x900000),
             dwq=D([W], ptr=0xa00000), dwk=D([W], ptr=0xa10000), eps=1e-6, flags=0, ws=None, ws_bytes=0)
    a.update(kw)
    return a


def norm_fwd(**kw):
    a = norm_args(**kw)
    return b.lib.mt_qk_norm_rope_fwd(*[R(a[n]) for n in ("q", "k", "wq", "wk", "cos", "sin", "yq", "yk")], a["eps"],
                                     a["flags"], None)


def norm_bwd(**kw):
    a = norm_args(**kw)
    return b.lib.mt_qk_norm_rope_bwd(*[R(a[n]) for n in ("q", "k", "wq", "wk", "cos", "sin", "yq", "yk", "dq", "dk",
                                                        "dwq", "dwk")], a["eps"], a["flags"], a["ws"], a["ws_bytes"],
                                     None)


@pytest.mark.parametrize("call", [norm_fwd, norm_bwd])
def test_norm_inputs(call):
    assert call(q=None) == NULL and call(yq=None) == NULL and call(yk=None) == NULL and call(sin=None) == NULL
    assert call(k=None, yk=None, dk=None, dwk=None) == NULL               # wk without k
    assert call(q=D([B, TQ, W], ptr=0x100000)) == NDIM
    assert call(yq=heads(TQ, HK, 0x600000)) == SHAPE
    assert call(k=heads(TK, HK, 0x200000), yk=heads(TK, HK, 0x700000)) == SHAPE
    assert call(k=heads(TQ, HK, 0x200000, BF16)) == DTYPE and call(yk=heads(TQ, HK, 0x700000, BF16)) == DTYPE
    assert call(wq=D([W - 1], ptr=0x300000)) == SHAPE and call(wk=D([W], BF16, 0x310000)) == DTYPE
    assert call(cos=D([B, TQ, W // 2], BF16, 0x400000)) == DTYPE
    assert call(cos=D([1, TQ, W // 2], ptr=0x400000)) == SHAPE
    assert call(cos=D([B, TQ, W // 4], ptr=0x400000)) == SHAPE            # not sin's
    assert call(cos=D([B, TQ, W], ptr=0x400000), sin=D([B, TQ, W], ptr=0x500000)) == SHAPE  # more pairs than W / 2
    assert call(cos=D([B, TQ, W // 2], ptr=0x400000, stride=[0, 0, 2])) == LAYOUT
    assert call(eps=-1.0) == INVALID and call(eps=math.nan) == INVALID and call(flags=8) == INVALID
    wide = dict(q=heads(TQ, HQ, 0x100000, width=1025), yq=heads(TQ, HQ, 0x600000, width=1025), k=None, yk=None, wk=None,
                dk=None, dwk=None, wq=None)
    assert call(**wide) == SHAPE


def test_norm_outputs():
    assert norm_fwd(flags=1) == INVALID
    assert norm_fwd(yq=heads(TQ, HQ, 0x100000)) == ALIAS and norm_fwd(yk=heads(TQ, HK, 0x600000)) == ALIAS
    assert norm_fwd(yq=heads(TQ, HQ, 0x600000, stride=[0, HQ * W, W, 1])) == LAYOUT
    assert norm_bwd(dq=None) == NULL and norm_bwd(dq=None, dk=None, dwq=None, dwk=None) == NULL
    assert norm_bwd(k=None, yk=None, wk=None, dk=None) == NULL            # dwk without k
    assert norm_bwd(dq=heads(TQ, HQ, 0x800000, BF16)) == DTYPE and norm_bwd(dwq=D([W], BF16, 0xa00000)) == DTYPE
    assert norm_bwd(dq=heads(TQ, HQ, 0x600000)) == ALIAS and norm_bwd(dwk=D([W], ptr=0xa00004)) == ALIAS
    assert norm_bwd() == WS and norm_bwd(ws=0x1000000, ws_bytes=16) == WS and norm_bwd(ws=0x1000001, ws_bytes=1 << 20) == WS


def test_dropout():
    X, Y, S = D([8, 6], ptr=0x10000), D([8, 6], ptr=0x20000), D([8, 6], ptr=0x30000)
    fw = lambda x, r, p, y: b.lib.mt_dropout_fwd(R(x), R(r), p, 1, 2, R(y), None)
    bw = lambda dy, p, dx, flags=0: b.lib.mt_dropout_bwd(R(dy), p, 1, 2, R(dx), flags, None)
    assert fw(None, S, 0.1, Y) == NULL and fw(X, S, 0.1, None) == NULL and bw(None, 0.1, Y) == NULL
    assert fw(D([48], ptr=0x10000), S, 0.1, Y) == NDIM
    assert fw(X, D([8, 5], ptr=0x30000), 0.1, Y) == SHAPE and fw(X, S, 0.1, D([7, 6], ptr=0x20000)) == SHAPE
    assert fw(X, D([8, 6], BF16, 0x30000), 0.1, Y) == DTYPE and fw(D([8, 6], I32, 0x10000), None, 0.1, Y) == DTYPE
    for bad in (-0.1, 1.1, math.nan, math.inf):
        assert fw(X, S, bad, Y) == INVALID and bw(X, bad, Y) == INVALID
    assert fw(X, S, 0.1, D([8, 6], ptr=0x20000, stride=[1, 8])) == LAYOUT
    assert fw(X, S, 0.1, D([8, 6], ptr=0x20000, stride=[5, 1])) == LAYOUT
    assert fw(X, S, 0.1, D([8, 6], ptr=0x10004)) == ALIAS and fw(X, S, 0.1, D([8, 6], ptr=0x30004)) == ALIAS
    assert bw(X, 0.1, Y, 2) == INVALID and bw(X, 0.1, D([8, 6], ptr=0x10000)) == ALIAS


def test_the_binding_refuses_what_it_cannot_describe():
    t = torch.zeros(1, 2, 2, 8)
    with pytest.raises(ValueError, match="device tensors"):
        b.attention_fwd(t, t, t, t)
    with pytest.raises(ValueError, match="device tensors"):
        b.attention_bwd(t, t, t, t, t, t, t)
    with pytest.raises(ValueError, match="device tensors"):
        b.qk_norm_rope_fwd(t, None, None, None, None, None, t, None)
    with pytest.raises(ValueError, match="device tensors"):
        b.dropout_fwd(t, None, 0.1, 1, 2, t)
    with pytest.raises(b.MtError):
        b.dropout_fwd(None, None, 0.1, 1, 2, None, stream=0)
    with pytest.raises(OverflowError):
        b.dropout_fwd(None, None, 0.1, -1, 2, None, stream=0)

    class Lengths:
        is_cuda, dtype = True, torch.int64

    with pytest.raises(TypeError, match="int32"):
        b.attention_fwd(None, None, None, None, kv_len=Lengths(), scale=1.0, stream=0)

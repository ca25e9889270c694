"""Host-side validation of the embedding, the layer norm, the cross-entropy loss and gradient clipping: every bad
argument is reported with the documented status before any HIP call. No case here passes validation, so nothing is ever
launched and no GPU is needed."""
import ctypes
import math

import pytest
import torch

from helpers import load_binding

b = load_binding()

from test_abi_host import BF16, D, F32, R  # noqa: E402

I32 = b.I32
NULL, NDIM, SHAPE, DTYPE, LAYOUT, ALIAS, WS, INVALID = 1, 2, 3, 4, 5, 6, 7, 9
WORK = 0x8000000
BIG = 1 << 30
M, V, W = 12, 50, 16


def caller(fn, names, **defaults):
    """A call of fn whose arguments are the defaults, some replaced by name."""
    def call(**kw):
        a = dict(defaults, **kw)
        assert set(a) == set(names), set(a) ^ set(names)
        return fn(*[R(a[n]) if isinstance(a[n], b.MtTensor) else a[n] for n in names])
    return call


ids = lambda *shape, ptr=0x100000, stride=None, dtype=I32: D(list(shape), dtype, ptr, stride)

emb_fwd = caller(b.lib.mt_embedding_fwd, ("ids", "table", "scale", "y", "stream"), ids=ids(M), table=D([V, W], ptr=0x200000),
                 scale=2.0, y=D([M, W], ptr=0x300000), stream=None)
emb_bwd = caller(b.lib.mt_embedding_bwd, ("ids", "dy", "scale", "dtable", "flags", "ws", "ws_bytes", "stream"), ids=ids(M),
                 dy=D([M, W], ptr=0x200000), scale=2.0, dtable=D([V, W], ptr=0x300000), flags=0, ws=WORK, ws_bytes=BIG,
                 stream=None)


@pytest.mark.parametrize("call", [emb_fwd, emb_bwd])
def test_tokens(call):
    assert call(ids=None) == NULL and call(ids=ids(M, ptr=0)) == NULL
    assert call(ids=ids(M, dtype=F32)) == DTYPE
    assert call(ids=ids()) == NDIM and call(ids=ids(2, 3, 2)) == NDIM
    assert call(ids=ids(M + 1)) == SHAPE and call(ids=ids(-1)) == SHAPE and call(ids=ids(3, 5)) == SHAPE
    assert call(ids=ids(M, stride=[-1])) == LAYOUT
    assert call(ids=ids((1 << 30) + 1)) == SHAPE and call(ids=ids(1 << 20, 1 << 20)) == SHAPE
    for bad in (math.nan, math.inf):
        assert call(scale=bad) == INVALID


def test_embedding():
    assert emb_fwd(table=None) == NULL and emb_fwd(y=None) == NULL
    assert emb_fwd(table=D([V, W, 1], ptr=0x200000)) == NDIM
    assert emb_fwd(table=D([V, W], I32, 0x200000)) == DTYPE and emb_fwd(y=D([M, W], I32, 0x300000)) == DTYPE
    assert emb_fwd(table=D([V, W + 1], ptr=0x200000)) == SHAPE and emb_fwd(y=D([M + 1, W], ptr=0x300000)) == SHAPE
    assert emb_fwd(table=D([V, W], ptr=0x200000, stride=[1, V])) == LAYOUT
    assert emb_fwd(y=D([M, W], ptr=0x300000, stride=[W - 1, 1])) == LAYOUT
    wide = (1 << 20) + 1
    assert emb_fwd(table=D([1, wide], ptr=0x20000000), y=D([M, wide], ptr=0x40000000)) == SHAPE
    assert emb_fwd(y=D([M, W], ptr=0x200000)) == ALIAS and emb_fwd(y=D([M, W], ptr=0x100000)) == ALIAS
    assert emb_fwd(ids=ids(M, ptr=0x300000 + 4 * M * W - 4)) == ALIAS


def test_embedding_gradient():
    assert emb_bwd(dy=None) == NULL and emb_bwd(dtable=None) == NULL
    assert emb_bwd(dtable=D([V, W], BF16, 0x300000)) == DTYPE and emb_bwd(dy=D([M, W], I32, 0x200000)) == DTYPE
    assert emb_bwd(dy=D([M, W + 1], ptr=0x200000)) == SHAPE and emb_bwd(dy=D([M - 1, W], ptr=0x200000)) == SHAPE
    assert emb_bwd(dtable=D([V, W], ptr=0x300000, stride=[W - 1, 1])) == LAYOUT
    assert emb_bwd(dy=D([M, W], ptr=0x200000, stride=[1, M])) == LAYOUT
    assert emb_bwd(dtable=D([(1 << 24) + 1, 1], ptr=0x20000000), dy=D([M, 1], ptr=0x200000)) == SHAPE
    many = (1 << 26) + 1
    assert emb_bwd(ids=ids(many, ptr=0x40000000), dy=D([many, 1], ptr=0x80000000), dtable=D([V, 1], ptr=0x300000)) == SHAPE
    assert emb_bwd(dtable=D([V, W], ptr=0x200000)) == ALIAS and emb_bwd(dtable=D([V, W], ptr=0x100000)) == ALIAS
    assert emb_bwd(flags=2) == INVALID and emb_bwd(flags=8) == INVALID
    assert emb_bwd(ws=None, ws_bytes=0) == WS and emb_bwd(ws_bytes=255) == WS and emb_bwd(ws=WORK + 16) == WS


norm_fwd = caller(b.lib.mt_layer_norm_fwd, ("x", "w", "b", "eps", "y", "stream"), x=D([M, W], ptr=0x100000),
                  w=D([W], ptr=0x200000), b=D([W], ptr=0x210000), eps=1e-5, y=D([M, W], ptr=0x300000), stream=None)
norm_bwd = caller(b.lib.mt_layer_norm_bwd, ("x", "w", "dy", "eps", "dx", "dw", "db", "flags", "ws", "ws_bytes", "stream"),
                  x=D([M, W], ptr=0x100000), w=D([W], ptr=0x200000), dy=D([M, W], ptr=0x300000), eps=1e-5,
                  dx=D([M, W], ptr=0x400000), dw=D([W], ptr=0x500000), db=D([W], ptr=0x510000), flags=0, ws=WORK,
                  ws_bytes=BIG, stream=None)


@pytest.mark.parametrize("call", [norm_fwd, norm_bwd])
def test_layer_norm_inputs(call):
    assert call(x=None) == NULL and call(x=D([M, W], ptr=0)) == NULL
    assert call(x=D([M * W], ptr=0x100000)) == NDIM
    assert call(x=D([M, W], I32, 0x100000)) == DTYPE and call(w=D([W], BF16, 0x200000)) == DTYPE
    assert call(x=D([M, 0], ptr=0x100000)) == SHAPE and call(x=D([M, 16385], ptr=0x100000)) == SHAPE
    assert call(w=D([W + 1], ptr=0x200000)) == SHAPE and call(w=D([W], ptr=0x200000, stride=[2])) == LAYOUT
    assert call(x=D([M, W], ptr=0x100000, stride=[1, M])) == LAYOUT
    for bad in (-1e-9, math.nan, math.inf):
        assert call(eps=bad) == INVALID


def test_layer_norm_outputs():
    assert norm_fwd(y=None) == NULL and norm_fwd(b=D([W + 1], ptr=0x210000)) == SHAPE
    assert norm_fwd(y=D([M, W + 1], ptr=0x300000)) == SHAPE and norm_fwd(y=D([M + 1, W], ptr=0x300000)) == SHAPE
    assert norm_fwd(y=D([M, W], ptr=0x300000, stride=[W - 1, 1])) == LAYOUT
    for at in (0x100000, 0x200000, 0x210000):
        assert norm_fwd(y=D([M, W], ptr=at)) == ALIAS
    assert norm_bwd(dy=None) == NULL and norm_bwd(dx=None, dw=None, db=None) == NULL
    assert norm_bwd(dy=D([M, W - 1], ptr=0x300000)) == SHAPE and norm_bwd(dx=D([M - 1, W], ptr=0x400000)) == SHAPE
    assert norm_bwd(dx=D([M, W], BF16, 0x400000)) == DTYPE          # not dy's
    assert norm_bwd(dw=D([W], BF16, 0x500000)) == DTYPE and norm_bwd(db=D([W - 1], ptr=0x510000)) == SHAPE
    assert norm_bwd(dx=D([M, W], ptr=0x300000)) == ALIAS and norm_bwd(dw=D([W], ptr=0x400000)) == ALIAS
    assert norm_bwd(db=D([W], ptr=0x500000)) == ALIAS and norm_bwd(dw=D([W], ptr=0x200000)) == ALIAS
    assert norm_bwd(flags=2) == INVALID
    assert norm_bwd(ws=None, ws_bytes=0) == WS and norm_bwd(ws_bytes=2 * W * 4 - 1) == WS and norm_bwd(ws=WORK + 4) == WS


xent = caller(b.lib.mt_cross_entropy, ("logits", "targets", "loss", "losses", "dlogits", "ws", "ws_bytes", "stream"),
              logits=D([M, V], ptr=0x100000), targets=ids(M, ptr=0x200000), loss=D([1], ptr=0x300000),
              losses=D([M], ptr=0x310000), dlogits=D([M, V], ptr=0x400000), ws=WORK, ws_bytes=BIG, stream=None)


def test_cross_entropy():
    assert xent(logits=None) == NULL and xent(targets=None) == NULL and xent(loss=None, losses=None, dlogits=None) == NULL
    assert xent(logits=D([M, V, 1], ptr=0x100000)) == NDIM and xent(logits=D([M, V], I32, 0x100000)) == DTYPE
    assert xent(logits=D([M, 0], ptr=0x100000)) == SHAPE and xent(logits=D([M, (1 << 24) + 1], ptr=0x100000)) == SHAPE
    assert xent(logits=D([M, V], ptr=0x100000, stride=[1, M])) == LAYOUT
    assert xent(targets=ids(M, ptr=0x200000, dtype=F32)) == DTYPE and xent(targets=ids(M + 1, ptr=0x200000)) == SHAPE
    assert xent(targets=ids(2, 5, ptr=0x200000)) == SHAPE and xent(targets=ids(2, 3, 2, ptr=0x200000)) == NDIM
    assert xent(loss=D([2], ptr=0x300000)) == SHAPE and xent(loss=D([1], BF16, 0x300000)) == DTYPE
    assert xent(losses=D([M + 1], ptr=0x310000)) == SHAPE and xent(losses=D([M], BF16, 0x310000)) == DTYPE
    assert xent(losses=D([M], ptr=0x310000, stride=[2])) == LAYOUT
    assert xent(dlogits=D([M, V - 1], ptr=0x400000)) == SHAPE and xent(dlogits=D([M, V], I32, 0x400000)) == DTYPE
    assert xent(dlogits=D([M, V], ptr=0x400000, stride=[V - 1, 1])) == LAYOUT
    assert xent(dlogits=D([M, V], ptr=0x100000)) == ALIAS and xent(dlogits=D([M, V], BF16, 0x200000)) == ALIAS
    assert xent(loss=D([1], ptr=0x310004)) == ALIAS and xent(losses=D([M], ptr=0x400000)) == ALIAS
    assert xent(loss=D([1], ptr=0x200004)) == ALIAS
    assert xent(ws=None, ws_bytes=0) == WS and xent(ws_bytes=100) == WS and xent(ws=WORK + 128) == WS


def clip(grads, out=None, most=1.0, norm=D([1], ptr=0x900000), ws=WORK, ws_bytes=BIG, n=None):
    arr = lambda ts: None if ts is None else (b.MtTensor * max(1, len(ts)))(*ts)
    return b.lib.mt_clip_grad_norm(len(grads) if n is None else n, None if n == 3 and not grads else arr(grads), most, arr(out),
                                   R(norm), ws, ws_bytes, None)


def test_clipping():
    A, B = D([8, 6], ptr=0x100000), D([5], BF16, 0x200000)
    assert clip([], n=-1) == INVALID and clip([], n=3) == NULL
    assert clip([A, D([5], BF16, 0)]) == NULL and clip([A, D([5], I32, 0x200000)]) == DTYPE
    assert clip([D([8, 6], ptr=0x100000, stride=[7, 1]), B]) == LAYOUT and clip([D([8, 6], ptr=0x100000, stride=[1, 8])]) == LAYOUT
    assert clip([D([-6], ptr=0x100000)]) == SHAPE
    for bad in (-1.0, -math.inf, math.nan):
        assert clip([A, B], most=bad) == INVALID
    assert clip([A, B], norm=D([2], ptr=0x900000)) == SHAPE and clip([A, B], norm=D([1], BF16, 0x900000)) == DTYPE
    # what is written overlaps nothing
    assert clip([A, A]) == ALIAS and clip([A, D([3], ptr=0x100000 + 4 * 47)]) == ALIAS
    assert clip([A, B], norm=D([1], ptr=0x100004)) == ALIAS
    X, Y = D([8, 6], BF16, 0x300000), D([5], ptr=0x400000)
    assert clip([A, B], [X, D([6], ptr=0x400000)]) == SHAPE and clip([A, B], [D([6, 8], ptr=0x300000), Y]) == SHAPE
    assert clip([A, B], [D([48], ptr=0x300000), Y]) == SHAPE
    assert clip([A, B], [X, D([5], ptr=0x400000, stride=[2])]) == LAYOUT and clip([A, B], [X, D([5], I32, 0x400000)]) == DTYPE
    assert clip([A, B], [A, Y]) == ALIAS and clip([A, B], [X, D([5], ptr=0x100000 + 4 * 47)]) == ALIAS
    assert clip([A, B], [X, D([5], ptr=0x300000)]) == ALIAS and clip([A, B], [X, Y], norm=D([1], ptr=0x400000)) == ALIAS
    assert clip([A, B], [X, Y], norm=D([1], ptr=0x200000)) == ALIAS
    # gradients that share memory are read only where others are written: the next check refuses
    assert clip([A, A], [X, D([8, 6], ptr=0x500000)], ws=None) == WS
    assert clip([A, B], ws=None, ws_bytes=0) == WS and clip([A, B], ws_bytes=4) == WS and clip([A, B], ws=WORK + 8) == WS


def test_clipping_of_sizes_whose_product_overflows():
    """2^64 values are not none: in 64 bits the product wraps to 0."""
    wide = 1 << 32
    for shape in ([wide, wide], [wide, wide, 3], [1 << 22] * 3, [1 << 40, 2], [(1 << 40) + 1]):
        t = D(shape, ptr=0x100000)
        assert clip([t]) == SHAPE and clip([D([5], ptr=0x200000)], [t]) == SHAPE
        assert b.lib.mt_clip_grad_norm_workspace(1, R(t), ctypes.byref(ctypes.c_size_t())) == SHAPE
    assert clip([D([5], ptr=0x200000)], norm=D([wide, wide], ptr=0x900000)) == SHAPE
    for norm in (D([wide, wide], ptr=0x100000), D([1 << 31, 1 << 31, 4], ptr=0x100000)):
        assert b.lib.mt_mse_loss(R(norm), R(norm), R(D([1], ptr=0x900000)), None, None, 0, None) == SHAPE


def test_clipping_of_empty_tensors():
    """A tensor without values is contiguous whatever its strides are (torch gives [5, 0] the strides 1 and 1), and without
    data; sizes beside the 0 do not overflow."""
    for shape, stride in (([0], [1]), ([0, 5], [5, 1]), ([5, 0], [1, 1]), ([5, 0], [0, 1]), ([3, 0, 7], [7, 7, 1]),
                          ([1 << 40, 1 << 40, 0], [9, 9, 1])):
        t = D(shape, ptr=0, stride=stride)
        assert clip([t], norm=None) == 0 and clip([t], [D(shape, BF16, 0, stride)], norm=None) == 0
        assert clip([t, D([5], ptr=0x200000)], ws_bytes=4) == WS  # the next check
        assert clip([t], norm=None, ws_bytes=4) == WS
    assert clip([D([5, 0], ptr=0, stride=[-1, 1])]) == LAYOUT and clip([D([-5, 0], ptr=0)]) == SHAPE
    assert clip([D([5, 0], I32, 0)]) == DTYPE
    assert clip([D([5, 0], ptr=0)], [D([0, 5], ptr=0)]) == SHAPE


def test_workspaces():
    n = ctypes.c_size_t()
    ask = lambda f, *a: f(*[R(t) if isinstance(t, b.MtTensor) else t for t in a], ctypes.byref(n))
    f = b.lib.mt_embedding_bwd_workspace
    tok, dy, dt = ids(M), D([M, W], ptr=0x200000), D([V, W], ptr=0x300000)
    assert ask(f, tok, dy, dt) == 0 and n.value >= 8 * M and n.value % 256 == 0
    assert ask(f, tok, dy, D([V, W], BF16, 0x300000)) == DTYPE and f(R(tok), R(dy), R(dt), None) == NULL
    assert ask(f, ids(0), D([0, W]), dt) == 0 and ask(f, tok, dy, D([0, W])) == 0
    f = b.lib.mt_layer_norm_bwd_workspace
    x, g, dw = D([M, W], ptr=0x100000), D([M, W], ptr=0x300000), D([W], ptr=0x500000)
    assert ask(f, x, None, g, None, dw, None) == 0 and n.value >= 8 * W
    assert ask(f, x, None, g, D([M, W], ptr=0x400000), None, None) == 0 and n.value == 0
    assert ask(f, x, None, g, None, None, None) == NULL and f(R(x), None, R(g), None, R(dw), None, None) == NULL
    f = b.lib.mt_cross_entropy_workspace
    z, t = D([M, V], ptr=0x100000), ids(M, ptr=0x200000)
    assert ask(f, z, t) == 0 and n.value >= 4 * M + 4
    assert ask(f, z, ids(M + 1, ptr=0x200000)) == SHAPE and f(R(z), R(t), None) == NULL
    f = b.lib.mt_clip_grad_norm_workspace
    two = (b.MtTensor * 2)(D([8, 6], ptr=0x100000), D([5], BF16, 0x200000))
    assert f(2, two, ctypes.byref(n)) == 0 and n.value >= 8
    assert f(0, None, ctypes.byref(n)) == 0 and n.value >= 8
    assert f(2, two, None) == NULL and f(-1, two, ctypes.byref(n)) == INVALID


def test_the_binding_refuses_what_it_cannot_describe():
    t = torch.zeros(2, 2)
    for call in (lambda: b.embedding_fwd(t, t, t), lambda: b.embedding_bwd(t, t, t), lambda: b.layer_norm_fwd(t, None, None, t),
                 lambda: b.layer_norm_bwd(t, None, t, t), lambda: b.cross_entropy(t, t, t), lambda: b.clip_grad_norm([t], 1.0),
                 lambda: b.embedding_bwd_workspace(t, t, t), lambda: b.layer_norm_bwd_workspace(t, None, t, t),
                 lambda: b.cross_entropy_workspace(t, t), lambda: b.clip_grad_norm_workspace([t])):
        with pytest.raises(ValueError, match="device tensors"):
            call()
    with pytest.raises(AssertionError, match="lengths"):
        b.clip_grad_norm([], 1.0, out=[t])
    with pytest.raises(TypeError):
        b.clip_grad_norm((x for x in [t]), 1.0)
    with pytest.raises(b.MtError, match="max_norm"):
        b.clip_grad_norm([], -1.0, stream=0)

    class Tokens:
        is_cuda, dtype = True, torch.int64

    for call in (lambda: b.embedding_fwd(Tokens(), None, None, stream=0), lambda: b.cross_entropy(None, Tokens(), stream=0)):
        with pytest.raises(TypeError, match="int32"):
            call()

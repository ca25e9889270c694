"""Which sizes, scales and packings attention's validation lets through, seen from the refusal that comes next: no case passes validation, so
nothing is launched and no GPU is needed."""
from helpers import load_binding

b = load_binding()

from test_abi_host import BF16, D, F32  # noqa: E402
from test_abi_host_attention import ALIAS, INVALID, SHAPE, WS, bwd, fwd  # noqa: E402


def test_scales():
    """2^-100 to 2^100: past the ends lse / scale, or scale in base 2, could pass the largest float."""
    for call in (fwd, bwd):
        for bad in (2.0 ** -101, 1e-37, 1e-40, 2.0 ** 101, 3e38):
            assert call(scale=bad) == INVALID
    for good in (2.0 ** -100, 0.125, 1.0, 2.0 ** 100):
        assert bwd(scale=good, ws=None, ws_bytes=0) == WS


def many(TQ, HQ, HK, TK=64, B=1, W=8):
    """A call of many rows whose first output lies on its queries."""
    q = D([B, TQ, HQ, W], BF16, 0x100000000000)
    k, v = (D([B, TK, HK, W], BF16, 0x200000000000 * i) for i in (1, 2))
    stats = D([B, HQ, TQ], F32, 0x300000000000)
    kw = dict(q=q, k=k, v=v, o=q, lse=stats)
    return [fwd(**kw), bwd(**kw, dout=D([B, TQ, HQ, W], BF16, 0x500000000000), dq=q, dk=None, dv=None)]


def test_rows():
    """Blocks of 128 tokens and heads, fewer than 2^23, are what bounds a call; its rows are not."""
    for size in ((1 << 20, 32, 1), (1 << 24, 8, 8), ((1 << 23) * 127, 1, 1)):
        assert many(*size) == [ALIAS, ALIAS], size
    for size in ((1 << 30, 1, 1), (1 << 25, 32, 1), (1, 1 << 23, 1)):
        assert many(*size) == [SHAPE, SHAPE], size
    assert many(1, 1, 1, TK=1 << 30) == [SHAPE, SHAPE] and many(1, 1, 1, TK=(1 << 23) * 127) == [ALIAS, ALIAS]


def test_heads_side_by_side_are_apart():
    """Each head's gradients next to one another in one buffer ([B, T, H, 3, W]) pass the overlap check; views that
    share a value, or reach into the next head, do not."""
    B, T, H, W = 2, 6, 4, 16
    view = lambda at, w=W, pitch=3 * W: D([B, T, H, w], F32, 0x700000 + 4 * at, [T * H * pitch, H * pitch, pitch, 1])
    q, k, v, o, dout = (D([B, T, H, W], F32, 0x100000 * (i + 1)) for i in range(5))
    call = lambda dq, dk, dv: bwd(q=q, k=k, v=v, o=o, dout=dout, lse=D([B, H, T], ptr=0x600000), dq=dq, dk=dk, dv=dv,
                                  ws=None)
    assert call(view(0), view(W), view(2 * W)) == WS
    assert call(view(2 * W), view(0), view(W)) == WS
    assert call(view(0), view(W - 1), view(2 * W)) == ALIAS
    assert call(view(0), view(W), view(2 * W + 1)) == ALIAS
    assert call(view(0), view(W, pitch=4 * W), view(2 * W)) == ALIAS
    assert call(view(0), view(W), view(3 * W)) == ALIAS  # the next head's dq

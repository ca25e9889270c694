"""Corners of attention and the head norms."""
import pytest
import torch

pytestmark = pytest.mark.gpu

from test_gpu_attention import DEV, backward, draw, forward  # noqa: E402


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

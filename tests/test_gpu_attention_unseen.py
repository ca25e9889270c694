"""Attention with infinities and NaN in places that take no part: keys that no query of the call sees, wherever the
causal edge lies in a tile, and queries that see no key."""
import math

import pytest
import torch

from attention_reference import check, reference

pytestmark = pytest.mark.gpu

from paper_2602_00125_amd import binding as b  # noqa: E402  (a missing library fails the module)
from test_gpu_attention import DEV, backward, draw, forward, splits  # noqa: E402,F401

NAMES = ("o", "lse", "dq", "dk", "dv")


def compare(got, ref):
    for name, t in zip(NAMES, got):
        check(name, t, *ref[name])


# (queries, keys, position of query 0 of each batch element): edges inside and at the ends of tiles of 32, 64 and 128
EDGES = [(10, 300, (90, 27)), (1, 200, (0, 130)), (150, 400, (101, 7)), (33, 128, (94, 95))]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("D", [64, 96, 128, 50])
@pytest.mark.parametrize("n", [-1, 0, 1, 3])
def test_keys_that_no_query_sees_may_hold_anything(dtype, D, n, splits):
    splits(n)
    for TQ, TK, starts in EDGES:
        q, k, v, dout = (draw((2, t, h, D), dtype, i) for i, (t, h) in enumerate(((TQ, 4), (TK, 2), (TK, 2), (TQ, 4))))
        for i, s in enumerate(starts):
            k[i, s + TQ:], v[i, s + TQ:] = math.nan, math.inf
        start = torch.tensor(starts, dtype=torch.int32, device=DEV)
        kw = dict(causal=True, q_start=start)
        o, lse = forward(q, k, v, **kw)
        grads = backward(q, k, v, o, lse, dout, **kw)
        # the reference leaves out what lies past a length
        compare((o, lse, *grads), reference(q, k, v, D ** -0.5, kv_len=start + TQ, dout=dout, **kw))
        for t in grads[1:]:
            for i, s in enumerate(starts):
                assert (t[i, s + TQ:] == 0).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("D", [64, 96, 128, 50])
@pytest.mark.parametrize("what", ["q", "dout"])
def test_queries_that_see_no_key_may_hold_anything(dtype, D, what):
    """Queries before every key: o = 0, lse = -inf, no gradient, and nothing of theirs in the keys' gradients."""
    TQ, TK = 150, 130
    starts = (-37, -149, -150, -64, 0)
    B = len(starts)
    q, k, v, dout = (draw((B, t, h, D), dtype, i) for i, (t, h) in enumerate(((TQ, 4), (TK, 2), (TK, 2), (TQ, 4))))
    kw = dict(causal=True, q_start=torch.tensor(starts, dtype=torch.int32, device=DEV))
    ref = reference(q, k, v, D ** -0.5, dout=dout, **kw)
    bad = q if what == "q" else dout
    for i, s in enumerate(starts):
        bad[i, :-s, ::2], bad[i, :-s, 1::2] = math.nan, math.inf
    o, lse = forward(q, k, v, **kw)
    grads = backward(q, k, v, o, lse, dout, **kw)
    compare((o, lse, *grads), ref)
    for i, s in enumerate(starts):
        assert (o[i, :-s] == 0).all() and (lse[i, :, :-s] == -math.inf).all() and (grads[0][i, :-s] == 0).all()

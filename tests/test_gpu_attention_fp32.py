"""How near fp32 attention is to 64 bits: what its products by three bf16 parts leave out.

u = 2^-24. With inputs drawn at random the errors of a result's terms have random signs, so that the error's norm is
that of the result times a term's: a probability's about 6 u (its score summed in 6 D / 16 roundings of at most u / 2,
the exponent's argument of up to 10 bits, the exponential), the sum's over up to 700 terms, 6 x 700 / 16 roundings,
about 5 u, and a gradient's twice in a row: 10 u or less. Four times that is the bar. Left-out parts are far past it:
with two parts a value, or three of the six products, at the sizes below, emulated in fp32, o is 70 to 840 u off,
dv 90 to 920, dq and dk 125 to 1240.
"""
import pytest
import torch

from attention_reference import reference

pytestmark = pytest.mark.gpu

from paper_2602_00125_amd import binding as b  # noqa: E402  (a missing library fails the module)
from test_gpu_attention import DEV, backward, draw, forward, splits  # noqa: E402,F401

U = 2.0 ** -24


@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("size", [(2, 64, 64, 2, 2, 64), (1, 257, 383, 2, 1, 112), (1, 509, 383, 4, 2, 128),
                                  (1, 700, 700, 1, 1, 128), (1, 128, 128, 8, 1, 80), (2, 60, 60, 2, 2, 50)], ids=str)
def test_error_of_random_data(size, causal, splits):
    B, TQ, TK, HQ, HK, D = size
    q, k, v, dout = (draw((B, t, h, D), "f32", i) for i, (t, h) in enumerate(((TQ, HQ), (TK, HK), (TK, HK), (TQ, HQ))))
    ref = reference(q, k, v, D ** -0.5, causal=causal, dout=dout)
    for n in (0, 1, 3):
        splits(n)
        o, lse = forward(q, k, v, causal=causal)
        grads = backward(q, k, v, o, lse, dout, causal=causal)
        for name, got in zip(("o", "lse", "dq", "dk", "dv"), (o, lse, *grads)):
            want = ref[name][0]
            some = want.isfinite()
            err = (got.double() - want)[some].norm() / want[some].norm()
            assert err <= 40 * U, f"{name} of {n} shares: {err / U:.1f} u"


@pytest.mark.parametrize("D", [16, 64, 128])
@pytest.mark.parametrize("sign", [1.0, -1.0])
def test_terms_left_out_of_a_product(D, sign, splits):
    """Queries and keys of one value whose lower parts are as large as they get (0x3f80ffff: cut off instead of rounded,
    its parts leave out 2^-21 of the product, 7.8 u). One key: lse is the score, D x^2, with the roundings of its
    conversion to base 2 and back, 1.3 u, and of the products' sums, at most 0.5 u for each of the three (of six) whose
    terms are not below u, and u / 2 a step of 16 d after the first, of random sign."""
    splits(0)
    x = torch.tensor([0x3F80FFFF], dtype=torch.int32).view(torch.float32).to(DEV)
    q, k = x.expand(1, 32, 1, D).contiguous(), sign * x.expand(1, 1, 1, D).contiguous()
    _, lse = forward(q, k, torch.ones_like(k), scale=1.0)
    want = sign * D * x.double() ** 2
    assert ((lse.double() - want).abs() <= (2.8 + 0.5 * (D / 16 - 1) ** 0.5) * U * want.abs()).all(), \
        ((lse.double() - want) / want / U).unique()

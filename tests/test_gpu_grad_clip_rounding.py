"""mt_clip_grad_norm's results in bf16 are rounded once."""
import numpy as np
import pytest
import torch

from language_reference import DEV, draw

pytestmark = pytest.mark.gpu

from paper_2602_00125_amd import binding as b  # noqa: E402  (a missing library fails the module)


def run(grads, max_norm, out):
    norm = torch.full((1,), float("nan"), device=DEV)
    ws = torch.full((b.clip_grad_norm_workspace(grads),), 0xff, dtype=torch.uint8, device=DEV)
    b.clip_grad_norm(grads, max_norm, norm, out=out, workspace=ws)


def to_bf16(v):
    """64-bit values to the nearest of 8 digits, ties to the even one (all in bf16's normal range)."""
    m, e = np.frexp(v)
    return np.ldexp(np.rint(m * 256.0), e - 8)


@pytest.mark.parametrize("source", ["f32", "bf16"])
def test_bf16_results_are_rounded_once(source):
    """A product that lies next to the middle of two bf16 values, closer than fp32 can tell, goes to its own side. The
    norm's 64-bit sum may be taken in another order here: that moves the factor by some 2^-52 of itself, and none of these
    products lies so near the middle (asserted)."""
    g = draw((1 << 22,), source, 1)
    for limit in (0.3, 700.0):
        out = torch.empty(g.shape, dtype=torch.bfloat16, device=DEV)
        run([g], limit, [out])
        v = g.double().cpu().numpy()
        v = v[np.abs(v) > 1e-30]
        f = limit / np.sqrt(np.sum(np.square(g.double().cpu().numpy())))
        got = out.double().cpu().numpy()[np.abs(g.double().cpu().numpy()) > 1e-30]
        want = to_bf16(v * f)
        sure = (to_bf16(v * f * (1 + 2.0 ** -48)) == want) & (to_bf16(v * f * (1 - 2.0 ** -48)) == want)
        assert sure.mean() > 0.999999
        assert np.array_equal(got[sure], want[sure])
        if source == "f32":  # and some of them tell the two apart
            twice = to_bf16((v * f).astype(np.float32).astype(np.float64))
            assert (twice != want)[sure].any()


def test_small_results():
    """Below bf16's normal range values are whole multiples of 2^-133, halves of them go to the even one, and signs,
    zeros and results that vanish are kept apart."""
    steps = np.array([0.0, -0.0, 0.25, -0.25, 0.5, -0.5, 0.50001, 0.75, 1.0, 1.49999, 1.5, 1.50001, 2.5, 100.5, -101.5, 0.4999999])
    g = torch.from_numpy(np.ldexp(steps, -127).astype(np.float32)).to(DEV)  # by the factor 2^-6 these are steps of 2^-133
    one = torch.tensor([1.0], device=DEV)
    out = [torch.full(t.shape, 9.0, dtype=torch.bfloat16, device=DEV) for t in (g, one)]
    run([g, one], 2.0 ** -6, out)  # the norm is 1: the squares of the others are below its last place
    want = np.ldexp(np.rint(np.ldexp(g.double().cpu().numpy(), 127)), -133)
    got = out[0].double().cpu().numpy()
    assert np.array_equal(got, want) and np.array_equal(np.signbit(got), np.signbit(want)) and out[1] == 2.0 ** -6

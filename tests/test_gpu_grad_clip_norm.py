"""mt_clip_grad_norm where the norm is past the range of fp32."""
import pytest
import torch

from language_reference import DEV, DT

pytestmark = pytest.mark.gpu

from paper_2602_00125_amd import binding as b  # noqa: E402  (a missing library fails the module)


def run(grads, max_norm, out=None):
    norm = torch.full((1,), float("nan"), device=DEV)
    ws = torch.full((b.clip_grad_norm_workspace(grads),), 0xff, dtype=torch.uint8, device=DEV)
    b.clip_grad_norm(grads, max_norm, norm, out=out, workspace=ws)
    return norm


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_a_norm_past_fp32_clips_nothing(dtype):
    """Of finite gradients: what norm holds is infinite, and by that the caller knows that nothing was clipped."""
    g = [torch.full((n,), 3e38, device=DEV).to(DT[dtype]) for n in (2, 5000)]
    keep = [t.clone() for t in g]
    assert run(g, 1.0) == float("inf") and all(torch.equal(a, c) for a, c in zip(g, keep))
    out = [torch.zeros_like(t) for t in g]
    assert run(g, 1.0, out) == float("inf") and all(torch.equal(a, c) for a, c in zip(out, keep))
    # the largest norm that fp32 holds clips
    one = [torch.full((1,), torch.finfo(torch.float32).max, device=DEV)]
    assert run(one, 2.0) == torch.finfo(torch.float32).max and one[0] == 2


def test_parameters_without_values():
    """Their gradients are clipped, and they are stepped, beside others, whatever strides torch gives them."""
    make = lambda: [torch.empty(5, 0, device=DEV), torch.full((4, 3), 2.0, device=DEV), torch.empty(3, 0, 7, device=DEV),
                    torch.empty(0, 6, device=DEV).T]
    grads, params, velocity = make(), make(), make()
    norm = run(grads, 1.0)
    assert abs(float(norm) - 48 ** 0.5) < 1e-5 and torch.allclose(grads[1], torch.full_like(grads[1], 12 ** -0.5))
    b.sgd_step(params, grads, velocity, 0.5)
    assert torch.equal(params[1], 2 - 0.5 * grads[1]) and torch.equal(velocity[1], grads[1])

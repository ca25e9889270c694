"""The example's block serves with the parameters that it has: after training steps, and before any pass."""
import pytest
import torch

pytestmark = pytest.mark.gpu

from test_gpu_attention_block import C, D, DEV, HK, HQ, AttentionBlock  # noqa: E402

T = 33


def decode_all(blk, x):
    """h of every token, one by one."""
    caches = [torch.full((2, T, HK, D), float("nan"), dtype=blk.dtype, device=DEV) for _ in range(2)]
    lens = torch.zeros(2, dtype=torch.int32, device=DEV)
    out = []
    for i in range(T):
        out.append(blk.decode(x[:, i].contiguous(), *caches, lens))
        lens += 1
    return torch.stack(out, 1)


@pytest.mark.parametrize("dtype,tol", [(torch.float32, 1e-5), (torch.bfloat16, 2e-2)])
@pytest.mark.parametrize("steps", [0, 1, 3])
def test_decoding_uses_the_parameters_of_the_last_step(dtype, tol, steps):
    """Tokens one by one against the whole sequence, computed after them. A step of Adam moves each weight by about
    lr = 0.05, a third of the largest: with the projections of before it the tokens are far off."""
    blk = AttentionBlock(2, T, C, HQ, HK, D, dtype, p=0.0, lr=0.05)
    g = torch.Generator("cpu")
    g.manual_seed(2)
    x, target = (torch.randn(2, T, C, generator=g).to(DEV) for _ in range(2))
    lens = torch.full((2,), T, dtype=torch.int32, device=DEV)
    for _ in range(steps):
        blk.step(x.view(-1, C), target.view(-1, C), lens)
    got = decode_all(blk, x).double()
    blk.forward(x.view(-1, C), lens)
    want = blk.h.view(2, T, C).double()
    assert (got - want).norm() <= tol * want.norm()

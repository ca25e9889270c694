"""The example's attention block: a training step against automatic differentiation in 64 bits, a falling loss, and
single tokens against a cache giving what the whole sequence gives."""
import os
import sys

import pytest
import torch

pytestmark = pytest.mark.gpu

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))

from attention_block import EPS, AttentionBlock, rotary_tables  # noqa: E402

DEV = "cuda:0"
B, T, C, HQ, HK, D = 3, 70, 48, 4, 2, 32


def inputs():
    g = torch.Generator("cpu")
    g.manual_seed(5)
    x, target = (torch.randn(B * T, C, generator=g).to(DEV) for _ in range(2))
    return x, target, torch.tensor([70, 41, 1], dtype=torch.int32, device=DEV)


def reference(blk, x, target, lens, mask):
    """h, the loss and the gradients of the parameters and x, in fp64."""
    P = {n: t.double().clone().requires_grad_() for n, t in blk.params.items()}
    X = x.double().clone().requires_grad_()
    qkv = (X @ P["wqkv"].T + P["bqkv"]).view(B, T, -1, D)
    cos, sin = (t.double()[:, None] for t in rotary_tables(torch.arange(T, device=DEV), D))

    def prepare(t, g):
        t = t * (t.square().mean(-1, keepdim=True) + EPS).rsqrt() * g
        a, b = t.chunk(2, -1)
        return torch.cat([a * cos - b * sin, b * cos + a * sin], -1)

    q, k, v = prepare(qkv[:, :, :HQ], P["gq"]), prepare(qkv[:, :, HQ:HQ + HK], P["gk"]), qkv[:, :, HQ + HK:]
    q, k, v = (t.permute(0, 2, 1, 3) for t in (q, k, v))
    k, v = (t.repeat_interleave(HQ // HK, 1) for t in (k, v))
    j = torch.arange(T, device=DEV)
    seen = (j[None] <= j[:, None])[None] & (j[None, None] < lens[:, None, None])
    S = torch.where(seen[:, None], q @ k.transpose(-1, -2) * D ** -0.5, -torch.inf)
    o = (S.softmax(-1) @ v).permute(0, 2, 1, 3).reshape(B * T, -1)
    h = X + mask * (o @ P["wo"].T + P["bo"])
    loss = (h - target.double()).square().mean()
    loss.backward()
    return h.detach(), loss.item(), {**{n: t.grad for n, t in P.items()}, "x": X.grad}


@pytest.mark.parametrize("dtype,tol", [(torch.float32, 2e-5), (torch.bfloat16, 3e-2)])
def test_step_against_automatic_differentiation(dtype, tol):
    """Normwise: fp32 sums of up to some hundred terms through four products; bf16 operands (2^-8 each) through
    eight roundings in a row."""
    blk = AttentionBlock(B, T, C, HQ, HK, D, dtype, p=0.25)
    x, target, lens = inputs()
    blk.forward(x, lens)
    ones = torch.ones_like(blk.y)
    mask = torch.empty_like(blk.y)
    from paper_2602_00125_amd import binding as mt
    mt.dropout_fwd(ones, None, blk.p, blk.seed, 0, mask)  # the mask times its scale
    params = {n: t.clone() for n, t in blk.params.items()}
    h, loss, grads = reference(blk, x, target, lens, mask.double())
    blk.step(x, target, lens)
    close = lambda a, b, what: (a.double() - b).norm() <= tol * b.norm() or pytest.fail(f"{what}: {(a.double() - b).norm() / b.norm():.2e}")
    close(blk.h, h, "h")
    assert abs(blk.loss.item() - loss) <= tol * loss
    for n, g in blk.grads.items():
        close(g, grads[n], n)
    close(blk.dx, grads["x"], "x")
    assert all((blk.params[n] != params[n]).any() for n in params)  # Adam has moved every parameter


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_the_loss_falls(dtype):
    blk = AttentionBlock(2, 128, 64, 4, 2, 32, dtype, lr=3e-3)
    g = torch.Generator("cpu")
    g.manual_seed(1)
    x = torch.randn(256, 64, generator=g).to(DEV)
    target = x + 0.5 * x.roll(1, -1)
    lens = torch.full((2,), 128, dtype=torch.int32, device=DEV)
    blk.step(x, target, lens)
    first = blk.loss.item()
    for _ in range(60):
        blk.step(x, target, lens)
    assert blk.loss.item() < 0.9 * first


@pytest.mark.parametrize("dtype,tol", [(torch.float32, 1e-5), (torch.bfloat16, 2e-2)])
def test_tokens_one_by_one_give_what_the_sequence_gives(dtype, tol):
    blk = AttentionBlock(2, 33, C, HQ, HK, D, dtype, p=0.0)
    x = torch.randn(2, 33, C, device=DEV)
    blk.forward(x.view(-1, C), torch.full((2,), 33, dtype=torch.int32, device=DEV))
    want = blk.h.view(2, 33, C).double()
    caches = [torch.full((2, 40, HK, D), float("nan"), dtype=dtype, device=DEV) for _ in range(2)]
    lens = torch.zeros(2, dtype=torch.int32, device=DEV)
    for i in range(33):
        h = blk.decode(x[:, i].contiguous(), *caches, lens)
        assert (h.double() - want[:, i]).norm() <= tol * want[:, i].norm(), i
        lens += 1

"""The example's language model: a training step's loss, norm and gradients against automatic differentiation in 64 bits,
single tokens against caches giving what the whole sequence gives, and a captured step."""
import os
import sys

import pytest
import torch

pytestmark = pytest.mark.gpu

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))

from attention_block import EPS, rotary_tables  # noqa: E402
from language_model import NORM_EPS, LanguageModel  # noqa: E402

from paper_2602_00125_amd import binding as mt  # noqa: E402

DEV = "cuda:0"
B, T, V, C, HQ, HK, D = 3, 37, 211, 48, 4, 2, 32


def make(layers, dtype, **kw):
    model = LanguageModel(V, layers, B, T, C, HQ, HK, D, dtype, **kw)
    g = torch.Generator("cpu")
    g.manual_seed(3)
    for n, t in model.params.items():  # norms that are not the identity
        if n != "table":
            t.add_((0.2 * torch.randn(t.shape, generator=g)).to(DEV))
    model.refresh()
    ids = torch.randint(0, V, (B, T), generator=g).to(DEV).int()
    targets = torch.randint(0, V, (B, T), generator=g).to(DEV).int()
    lens = torch.tensor([T, 20, 1], dtype=torch.int32, device=DEV)
    counts = torch.arange(T, device=DEV) < lens[:, None]
    return model, torch.where(counts, ids, -1), torch.where(counts, targets, -1), lens


def reference(model, ids, targets, lens):
    """logits, the loss and the gradients of all parameters, in fp64."""
    P = {n: t.double().clone().requires_grad_() for n, t in model.params.items()}
    Q = [{n: t.double().clone().requires_grad_() for n, t in b.params.items()} for b in model.blocks]
    norm = lambda x, i: (x - x.mean(-1, keepdim=True)) / (x.var(-1, unbiased=False, keepdim=True) + NORM_EPS).sqrt() * P[f"w{i}"] + P[f"b{i}"]
    cos, sin = (t.double()[:, None] for t in rotary_tables(torch.arange(T, device=DEV), D))
    j = torch.arange(T, device=DEV)
    seen = ((j[None] <= j[:, None])[None] & (j[None, None] < lens[:, None, None]))[:, None]

    def turn(t, g):
        t = t * (t.square().mean(-1, keepdim=True) + EPS).rsqrt() * g
        a, b = t.chunk(2, -1)
        return torch.cat([a * cos - b * sin, b * cos + a * sin], -1)

    h = torch.where((ids >= 0)[..., None], P["table"][ids.clamp(min=0).long()] * model.scale, 0.0).view(B * T, C)
    for i, q_ in enumerate(Q):
        qkv = (norm(h, i) @ q_["wqkv"].T + q_["bqkv"]).view(B, T, -1, D)
        q, k, v = turn(qkv[:, :, :HQ], q_["gq"]), turn(qkv[:, :, HQ:HQ + HK], q_["gk"]), qkv[:, :, HQ + HK:]
        q, k, v = (t.permute(0, 2, 1, 3) for t in (q, k, v))
        k, v = (t.repeat_interleave(HQ // HK, 1) for t in (k, v))
        S = torch.where(seen, q @ k.transpose(-1, -2) * D ** -0.5, -torch.inf)
        h = h + (S.softmax(-1) @ v).permute(0, 2, 1, 3).reshape(B * T, -1) @ q_["wo"].T + q_["bo"]
    logits = norm(h, len(Q)) @ P["table"].T
    t = targets.flatten().long()
    logp = logits.log_softmax(-1)[t >= 0]
    loss = -logp.gather(1, t[t >= 0][:, None]).mean()
    loss.backward()
    return logits.detach(), loss.item(), [t.grad for t in [*P.values(), *(t for q_ in Q for t in q_.values())]]


# Normwise. fp32: about 40 operations in a row, whose sums of up to some hundred terms are each off by up to 2e-6 of their
# norm. bf16, one layer: the operands of five products, the heads, P and their like in the gradient are rounded, twelve in
# a row (2^-8 each).
@pytest.mark.parametrize("layers,dtype,tol", [(2, torch.float32, 8e-5), (1, torch.bfloat16, 12 * 2.0 ** -8)])
def test_step_against_automatic_differentiation(layers, dtype, tol):
    model, ids, targets, lens = make(layers, dtype, max_norm=1e-3)
    logits, loss, grads = reference(model, ids, targets, lens)
    before = [t.clone() for t in model.all_params()]
    model.forward(ids, lens)
    model.backward(ids, targets, lens)
    close = lambda a, b, what: (a.double() - b).norm() <= tol * b.norm() or pytest.fail(f"{what}: {(a.double() - b).norm() / b.norm():.2e}")
    close(model.logits, logits, "logits")
    assert abs(model.loss.item() - loss) <= tol * loss
    names = [*model.params, *(f"{n}{i}" for i, b in enumerate(model.blocks) for n in b.params)]
    for name, got, want in zip(names, model.all_grads(), grads):
        close(got, want, name)
    model.step(ids, targets, lens)
    norm = sum(g.square().sum() for g in grads).sqrt()
    assert abs(model.norm.item() - norm) <= tol * norm
    clipped = sum(g.double().square().sum() for g in model.all_grads()).sqrt()
    assert abs(clipped.item() / 1e-3 - 1) < 1e-6
    assert all((a != b).any() for a, b in zip(model.all_params(), before))  # Adam has moved every parameter


@pytest.mark.parametrize("dtype,tol", [(torch.float32, 2e-5), (torch.bfloat16, 3e-2)])
def test_tokens_one_by_one_give_what_the_sequence_gives(dtype, tol):
    model, ids, _, _ = make(2, dtype)
    ids = ids.clamp(min=0)
    model.forward(ids, torch.full((B,), T, dtype=torch.int32, device=DEV))
    want = model.logits.view(B, T, V).double()
    caches = [[torch.full((B, T + 3, HK, D), float("nan"), dtype=dtype, device=DEV) for _ in range(2)] for _ in model.blocks]
    lens = torch.zeros(B, dtype=torch.int32, device=DEV)
    for i in range(T):
        got = model.decode(ids[:, i], caches, lens)
        assert (got.double() - want[:, i]).norm() <= tol * want[:, i].norm(), i
        lens += 1


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_a_captured_step_replays(dtype):
    """Forward, loss, backward and clipping in one graph: every replay gives the eager step's bits, on the batch that its
    buffers then hold, with eager work of the program in between."""
    model, ids, targets, lens = make(2, dtype, max_norm=1e-3)

    def run():
        model.forward(ids, lens)
        model.backward(ids, targets, lens)
        mt.clip_grad_norm(model.all_grads(), model.max_norm, model.norm, workspace=model.ws)
        return [model.loss, model.norm, model.logits, model.dlogits, *model.all_grads()]

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        run()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        outs = run()
    for r in range(4):
        ids.copy_(torch.where(ids >= 0, (ids + 7 * r) % V, -1))
        if r == 3:
            targets.fill_(-1)  # nothing counts
        eager = [t.clone() for t in run()]
        for t in outs:
            t.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(outs, eager)), r
    assert model.loss == 0 and model.norm == 0


def test_two_streams_at_once():
    """Two models, each on a stream of its own: the same results as one after the other."""
    runs = [make(1, torch.float32, seed=s) for s in (1, 2)]
    want = []
    for model, ids, targets, lens in runs:
        model.forward(ids, lens)
        model.backward(ids, targets, lens)
        want.append([model.loss.clone(), *(t.clone() for t in model.all_grads())])
    streams = [torch.cuda.Stream() for _ in runs]
    torch.cuda.synchronize()
    for _ in range(5):
        for s, (model, ids, targets, lens) in zip(streams, runs):
            with torch.cuda.stream(s):
                model.forward(ids, lens)
                model.backward(ids, targets, lens)
    torch.cuda.synchronize()
    for (model, *_), w in zip(runs, want):
        assert all(torch.equal(a, b) for a, b in zip([model.loss, *model.all_grads()], w))


def test_the_example_runs(monkeypatch, capsys):
    import language_model

    monkeypatch.setattr(sys, "argv", ["language_model.py", "--steps", "2", "--vocab", "501", "--batch", "2", "--tokens", "96",
                                      "--width", "64", "--heads", "2", "--kv-heads", "1", "--head-width", "32", "--dtype", "bf16"])
    language_model.main()
    assert "us a token" in capsys.readouterr().out

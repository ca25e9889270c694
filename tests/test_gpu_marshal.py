"""Tensors of every kind reach the library as they are: the binding reads plain ones by torch's exchange functions and
others by their attributes, and both describe the same memory."""
import pytest
import torch

pytestmark = pytest.mark.gpu

from paper_2602_00125_amd import binding as b  # noqa: E402  (a missing library fails the module)

DEV = "cuda:0"


class Sub(torch.Tensor):
    """Not a plain tensor: read by its attributes."""


def copy(x, y):
    b.dropout_fwd(x, None, 0.0, 0, 0, y)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_views(dtype):
    base = torch.randn(40, 60, device=DEV).to(dtype)
    for x in (base, base[3:, 5:], base[::3, 7:20], base[:1, :1], base[5:5], base[7].expand(12, 60), base[:, 9:10]):
        for kind in (lambda t: t, lambda t: t.as_subclass(Sub), torch.nn.Parameter, lambda t: t.detach().requires_grad_()):
            y = torch.full(x.shape, 9.0, dtype=dtype, device=DEV)
            copy(kind(x), y)
            assert torch.equal(y, x)


def test_workspaces_and_ranks():
    g = torch.randn(6, 5, 4, 3, 2, device=DEV)
    need = b.reduce_broadcast_grad_workspace(g, g[0, 0])
    for ws in (torch.empty(need + 4, dtype=torch.uint8, device=DEV), torch.empty(need // 8 + 1, dtype=torch.float64, device=DEV),
               torch.empty(need // 4 + 1, device=DEV).as_subclass(Sub), None):
        out = torch.empty(4, 3, 2, device=DEV)
        b.reduce_broadcast_grad(g, out, workspace=ws)
        assert (out - g.sum((0, 1))).abs().max() < 1e-5
    norm = torch.empty((), device=DEV)
    one = torch.full((), 3.0, device=DEV)
    b.clip_grad_norm([one], 1.0, norm, workspace=torch.empty(256, dtype=torch.uint8, device=DEV))
    assert norm == 3 and one == 1


def test_refusals():
    t = torch.zeros(2, 2, device=DEV)
    for bad in (t.double(), t.half(), t.int(), t.to_sparse(), torch.zeros((1,) * 9, device=DEV)):
        with pytest.raises((TypeError, ValueError, RuntimeError)):
            copy(bad, t)
    with pytest.raises(ValueError, match="device tensors"):
        copy(t, t.cpu())
    with pytest.raises(AssertionError, match="workspace"):
        b.linear_bwd(t, t, t, t.clone(), workspace=torch.empty(64))
    with pytest.raises(TypeError, match="int32"):
        b.embedding_fwd(t.long(), t, t.clone())


def test_tensors_of_another_device_are_refused():
    """With another current device than the tensors' (one card: the binding is told so) the newer calls refuse, unless
    their stream is given."""
    t, ids = torch.zeros(4, 4, device=DEV), torch.zeros(4, dtype=torch.int32, device=DEV)
    ws = torch.empty(1 << 16, dtype=torch.uint8, device=DEV)
    calls = [lambda **k: b.embedding_fwd(ids, t, t.clone(), **k), lambda **k: b.layer_norm_fwd(t, None, None, t.clone(), **k),
             lambda **k: b.embedding_bwd(ids, t, t.clone(), workspace=ws, **k), lambda **k: b.layer_norm_bwd(t, None, t, t.clone(), **k),
             lambda **k: b.cross_entropy(t, ids, losses=t[0].clone(), workspace=ws, **k),
             lambda **k: b.clip_grad_norm([t.clone()], 1.0, workspace=ws, **k)]
    for call in calls:
        call()
    b._m.init(*b._INIT[:-1], lambda: 1)
    try:
        for call in calls:
            with pytest.raises(ValueError, match="device"):
                call()
            call(stream=torch.cuda.current_stream())
    finally:
        b._m.init(*b._INIT)
    calls[0]()
    torch.cuda.synchronize()

"""mt_cross_entropy's sums: a row's exponentials, however many of them a thread meets, and the mean over many rows."""
import pytest
import torch

from language_reference import DEV, DT, U, close, cross_entropy, draw, integers

pytestmark = pytest.mark.gpu

from paper_2602_00125_amd import binding as b  # noqa: E402  (a missing library fails the module)


def run(z, t, dtype=None):
    loss, losses = torch.full((1,), float("nan"), device=DEV), torch.full((z.shape[0],), float("nan"), device=DEV)
    dz = None if dtype is None else torch.full(z.shape, float("nan"), dtype=DT[dtype], device=DEV)
    ws = torch.full((b.cross_entropy_workspace(z, t),), 0xff, dtype=torch.uint8, device=DEV)
    b.cross_entropy(z, t, loss, losses, dz, workspace=ws)
    return loss, losses, dz


@pytest.mark.parametrize("x", ["f32", "bf16"])
@pytest.mark.parametrize("V", [200003, 1 << 20, (1 << 22) + 5, 1 << 24])
def test_rows_of_many_logits(V, x):
    """The first logits are 0 and the others alike, so that every thread adds many equal exponentials, whose roundings have
    one sign. DEPTH (language_reference.py) holds for every length: 16 exponentials are added in fp32, sixteens in 64 bits,
    then 32 that a thread holds, 6 steps over the lanes and up to 16 waves: 71 roundings."""
    z = torch.tensor([[-1.234], [-0.3], [-2.0]], device=DEV).expand(3, V).to(DT[x]).contiguous()
    z[:, :65536] = 0.0
    t = torch.tensor([V // 3, 0, V - 1], dtype=torch.int32, device=DEV)
    got = run(z, t, "f32")
    for name, g, w in zip(("loss", "losses", "dlogits"), got, cross_entropy(z, t, torch.float32)):
        close(name, g, *w)


@pytest.mark.parametrize("x", ["f32", "bf16"])
@pytest.mark.parametrize("M,V", [(100000, 33), (1000, 10), (300, 40), (40000, 1025), (20000, 513), (3000, 5000)])
def test_the_mean_is_that_of_the_losses(M, V, x):
    """The losses are added in 64 bits and the mean is rounded once: half a step."""
    z, t = draw((M, V), x, 1, 2.0), integers((M,), -1, V, 2)
    n = int((t >= 0).sum())
    for out in (None, "bf16"):
        loss, losses, _ = run(z, t, out)
        assert not losses[t < 0].any()
        want = losses.double().sum() / n
        assert abs(float(loss) - float(want)) <= (U + 1e-12) * float(want)

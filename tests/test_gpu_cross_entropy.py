"""mt_cross_entropy against the formulas in 64 bits; the bounds are derived in language_reference.py."""
import pytest
import torch

from language_reference import DEV, DT, U, Apart, close, cross_entropy, draw, integers

pytestmark = pytest.mark.gpu

from paper_2602_00125_amd import binding as b  # noqa: E402  (a missing library fails the module)

TYPES = [("f32", "f32"), ("bf16", "bf16"), ("f32", "bf16"), ("bf16", "f32")]
INF = float("inf")


def run(z, t, dtype=None, loss=True, losses=True, dz=None):
    M, V = z.shape
    nan = lambda *shape: torch.full(shape, float("nan"), device=DEV)
    out = [nan(1) if loss else None, nan(M) if losses else None, dz]
    if dtype is not None and dz is None:
        out[2] = nan(M, V).to(dtype)
    ws = torch.full((b.cross_entropy_workspace(z, t),), 0xff, dtype=torch.uint8, device=DEV)
    b.cross_entropy(z, t, *out, workspace=ws)
    return out


def compare(got, want):
    for name, g, w in zip(("loss", "losses", "dlogits"), got, want):
        if g is not None:
            close(name, g, *w)


def targets(M, V, padded, seed=0):
    t = integers((M,), 0, V, seed)
    if padded:
        what = integers((M,), 0, 5, seed + 1)
        t = torch.where(what == 0, -1, torch.where(what == 1, V, t)).int()
    return t


SIZES = [(1, 1), (1, 2), (5, 10), (512, 10), (100, 8), (70, 9), (33, 64), (33, 65), (20, 511), (20, 512), (9, 513), (8, 1000),
         (7, 4097), (5, 16384), (5, 16385), (3, 32768), (3, 32771), (4, 50001), (2, 65536), (2, 65537), (1, 131072),
         (2, 200003), (2000, 37)]


@pytest.mark.parametrize("padded", [False, True])
@pytest.mark.parametrize("x,y", TYPES)
@pytest.mark.parametrize("M,V", SIZES)
def test_sizes(M, V, x, y, padded):
    z, t = draw((M, V), x, 1, 3.0), targets(M, V, padded, 2)
    if padded:  # rows that do not count may hold anything
        z[(t < 0) | (t >= V)] = float("nan")
    want = cross_entropy(z.nan_to_num(0.0), t, DT[y])
    got = run(z, t, DT[y])
    compare(got, want)
    for only in range(3):
        out = run(z, t, DT[y] if only == 2 else None, only == 0, only == 1)
        assert torch.equal(out[only], got[only])


@pytest.mark.parametrize("x,y", TYPES)
@pytest.mark.parametrize("V", [7, 100, 777, 2050, 70001])
def test_views(V, x, y):
    for off, extra in ((3, 5), (4, 4), (1, 0), (0, 3)):
        place = Apart(off, extra)
        z = place.inside(draw((6, V), x, 3, 2.0))
        t = targets(12, V, True, 4).view(3, 4)[:, ::2]  # [3, 2], strides 4 and 2
        dz = place.out(6, V, DT[y])
        compare(run(z, t, dz=dz), cross_entropy(z, t, DT[y]))
        place.check()
        t = targets(6, V, False, 5).view(2, 3).T
        compare(run(z, t, dz=dz), cross_entropy(z, t, DT[y]))
    same = draw((1, V), x, 6).expand(6, V)  # one row of logits for all
    t = targets(6, V, False, 7)
    compare(run(same, t, DT[y]), cross_entropy(same, t, DT[y]))


@pytest.mark.parametrize("V", [11, 1000, 66000])
@pytest.mark.parametrize("x", ["f32", "bf16"])
def test_masked_classes(V, x):
    """Logits of -infinity and of the type's lowest value have probability 0."""
    z, t = draw((8, V), x, 8, 2.0), targets(8, V, False, 9)
    gone = draw((8, V), "f32", 10) > 0.3
    gone[torch.arange(8), t.long()] = False
    z[gone] = -INF
    z[5, gone[5]] = torch.finfo(z.dtype).min
    z[6] = -INF
    z[6, t[6].long()] = 2.5  # the class alone is left
    got = run(z, t, torch.float32)
    compare(got, cross_entropy(z, t, torch.float32))
    assert not got[2][gone].any() and got[1][6] == 0 and not got[2][6].any()
    # the class itself is masked: infinite loss, the gradient that of a softmax
    z[2, t[2].long()] = -INF
    got = run(z, t, torch.float32)
    assert got[0] == INF and got[1][2] == INF
    close("dlogits", got[2], *cross_entropy(z, t, torch.float32)[2])


@pytest.mark.parametrize("V", [11, 1000, 66000])
def test_rows_that_have_no_softmax(V):
    z, t = draw((9, V), "f32", 11), targets(9, V, False, 12)
    z[1] = -INF
    z[3, V // 2] = INF
    z[4, V - 1] = float("nan")
    z[7] = float("nan")
    z[8] = -INF
    z[8, 3] = float("nan")
    bad, good = [1, 3, 4, 7, 8], [0, 2, 5, 6]
    loss, losses, dz = run(z, t, torch.float32)
    assert loss.isnan() and losses[bad].isnan().all() and dz[bad].isnan().all()
    # the others as they are without them
    z[bad] = 0.0
    want = cross_entropy(z, t, torch.float32)
    close("losses", losses[good], want[1][0][good], want[1][1][good])
    close("dlogits", dz[good], want[2][0][good], want[2][1][good])


@pytest.mark.parametrize("V", [40, 5000, 70000])
def test_far_apart_logits(V):
    """Differences past the range of exp; all alike; and large ones whose rounding must not grow in the exponential."""
    z, t = draw((6, V), "f32", 13), targets(6, V, False, 14)
    z[0] *= 1e30
    z[1] = 3e38
    z[2, :] = 12345.0
    z[3] += 30000.0
    z[4] = torch.linspace(-140, 0, V, device=DEV)
    z[5] = torch.linspace(0, -90, V, device=DEV)
    compare(run(z, t, torch.float32), cross_entropy(z, t, torch.float32))


def test_nothing_counts():
    z = torch.full((7, 30), float("nan"), device=DEV)
    loss, losses, dz = run(z, torch.full((7,), -1, dtype=torch.int32, device=DEV), torch.bfloat16)
    assert loss == 0 and not losses.any() and not dz.any()
    z = torch.empty((0, 30), device=DEV)
    loss, losses, dz = run(z, torch.empty((0,), dtype=torch.int32, device=DEV), torch.float32)
    assert loss == 0


@pytest.mark.parametrize("M,V", [(100000, 33), (30000, 600)])
def test_many_rows(M, V):
    z, t = draw((M, V), "f32", 15, 2.0), targets(M, V, True, 16)
    got = run(z, t, torch.float32)
    compare(got, cross_entropy(z, t, torch.float32))
    again = run(z, t, torch.float32)
    assert all(torch.equal(a, c) for a, c in zip(got, again))


@pytest.mark.parametrize("x,y", TYPES)
@pytest.mark.parametrize("V", [64, 65, 1024, 1025, 8192, 8193, 16384, 16385, 32768, 32769])
def test_where_the_forms_meet(V, x, y):
    """At the numbers of rows and logits where another way of sharing the work out begins."""
    for M in (256, 257, 512, 513):
        z, t = draw((M, V), x, 30, 2.0), targets(M, V, True, 31)
        compare(run(z, t, DT[y]), cross_entropy(z, t, DT[y]))


@pytest.mark.parametrize("V,L", [(1030, 1), (3, 256)])
def test_more_rows_than_blocks(V, L):
    """More rows than the blocks of a launch (2^20, of L rows each) hold at a time."""
    M = (1 << 20) * L + 300
    z = torch.zeros((M, V), dtype=torch.bfloat16, device=DEV)
    t = torch.full((M,), -1, dtype=torch.int32, device=DEV)
    at = torch.tensor([0, 5, (1 << 20) * L - 1, (1 << 20) * L, M - 1], device=DEV)
    z[at] = draw((5, V), "bf16", 20)
    t[at] = targets(5, V, False, 21)
    loss, losses, dz = run(z, t, torch.bfloat16)
    want = cross_entropy(z[at], t[at], torch.bfloat16)
    close("loss", loss, *want[0])
    close("losses", losses[at], *want[1])
    close("dlogits", dz[at], *want[2])
    assert torch.count_nonzero(losses) == 5 and torch.count_nonzero(dz.any(-1)) == 5


def test_gradient_against_differences():
    """Of the loss in 64 bits, by central differences, off by h^2 / 6 of a third derivative below 1."""
    z, t = draw((3, 9), "f32", 17), torch.tensor([2, -1, 8], dtype=torch.int32, device=DEV)
    dz = run(z, t, torch.float32)[2]
    h = 1e-4
    for m in range(3):
        for v in range(9):
            up, down = z.double().clone(), z.double().clone()
            up[m, v] += h
            down[m, v] -= h
            f = lambda x: float(cross_entropy(x, t, torch.float32)[0][0])
            assert abs((f(up) - f(down)) / (2 * h) - float(dz[m, v])) < h * h + 40 * U, (m, v)


def test_past_2_31_logits():
    M, V = 66000, 32771
    z = torch.zeros((M, V), dtype=torch.bfloat16, device=DEV)
    z[-2:] = draw((2, V), "bf16", 18)
    t = torch.full((M,), -1, dtype=torch.int32, device=DEV)
    t[0], t[-1], t[-2] = 5, V - 1, 0
    loss, losses, dz = run(z, t, torch.bfloat16)
    at = [0, M - 2, M - 1]
    want = cross_entropy(z[at], t[at], torch.bfloat16)
    close("loss", loss, *want[0])
    close("losses", losses[at], *want[1])
    close("dlogits", dz[at], *want[2])
    assert not losses[1:-2].any() and not dz[1:-2].any()

"""mt_layer_norm_fwd and mt_layer_norm_bwd against the formulas in 64 bits; the bounds are derived in
language_reference.py."""
import pytest
import torch

from language_reference import DEV, DT, Apart, close, draw, layer_norm, layer_norm_grad

pytestmark = pytest.mark.gpu

from paper_2602_00125_amd import binding as b  # noqa: E402  (a missing library fails the module)

TYPES = [("f32", "f32"), ("bf16", "bf16"), ("f32", "bf16"), ("bf16", "f32")]
EPS = 1e-5


def rows(M, C, dtype, seed):
    """Rows of different sizes and offsets."""
    x = draw((M, C), "f32", seed)
    scale = 10.0 ** (torch.arange(M, device=DEV) % 5 - 2)[:, None]
    return (x * scale + scale * (torch.arange(M, device=DEV) % 3)[:, None]).to(DT[dtype])


def weights(C, seed):
    return 1 + 0.2 * draw((C,), "f32", seed), draw((C,), "f32", seed + 1)


def new(M, C, dtype):
    return torch.full((M, C), float("nan"), dtype=DT[dtype] if isinstance(dtype, str) else dtype, device=DEV)


def run_bwd(x, w, dy, dx, dw, db, eps=EPS, accumulate=False):
    n = b.layer_norm_bwd_workspace(x, w, dy, dx, dw, db)
    ws = torch.full((n,), 0xff, dtype=torch.uint8, device=DEV) if n else None
    b.layer_norm_bwd(x, w, dy, dx, dw, db, eps=eps, accumulate=accumulate, workspace=ws)


SIZES = [(1, 1), (1, 4096), (7, 16384), (3, 16383), (64, 4096), (100, 1), (130, 3), (1000, 16), (33, 17), (257, 100),
         (50, 255), (50, 777), (9, 1025), (21, 2048), (5, 5000), (2, 8193), (700, 513), (40, 2560), (11, 2999), (13, 6144),
         (5, 7001), (4, 12288), (3, 10007)]


@pytest.mark.parametrize("x,y", TYPES)
@pytest.mark.parametrize("M,C", SIZES)
def test_forward(M, C, x, y):
    t = rows(M, C, x, 1)
    w, bias = weights(C, 2)
    for use in ((w, bias), (None, None)):
        out = new(M, C, y)
        b.layer_norm_fwd(t, *use, out, eps=EPS)
        close("y", out, *layer_norm(t, *use, EPS, DT[y]))


@pytest.mark.parametrize("x,y", TYPES)
@pytest.mark.parametrize("M,C", SIZES)
def test_gradients(M, C, x, y):
    t, dy = rows(M, C, x, 3), draw((M, C), y, 4)
    w, _ = weights(C, 5)
    dx, dw, db = new(M, C, y), new(1, C, "f32")[0], new(1, C, "f32")[0]
    run_bwd(t, w, dy, dx, dw, db)
    for name, got, want in zip(("dx", "dw", "db"), (dx, dw, db), layer_norm_grad(t, w, dy, EPS)):
        close(name, got, *want)
    # again, one at a time, without weights
    only = new(M, C, y)
    run_bwd(t, w, dy, only, None, None)
    assert torch.equal(only, dx)
    for k in range(2):
        part = [None, None]
        part[k] = new(1, C, "f32")[0]
        run_bwd(t, w, dy, None, *part)
        assert torch.equal(part[k], (dw, db)[k])
    run_bwd(t, None, dy, only, None, None)
    close("dx", only, *layer_norm_grad(t, None, dy, EPS)[0])


@pytest.mark.parametrize("x,y", TYPES)
@pytest.mark.parametrize("M,C", [(1, 8), (600, 40), (2000, 777), (40, 9000)])
def test_gradients_are_added(M, C, x, y):
    t, dy = rows(M, C, x, 6), draw((M, C), y, 7)
    w, _ = weights(C, 8)
    old = [draw((M, C), y, 9), draw((C,), "f32", 10), draw((C,), "f32", 11)]
    got = [o.clone() for o in old]
    run_bwd(t, w, dy, *got, accumulate=True)
    for name, g, want in zip(("dx", "dw", "db"), got, layer_norm_grad(t, w, dy, EPS, old)):
        close(name, g, *want)


@pytest.mark.parametrize("x,y", TYPES)
@pytest.mark.parametrize("C", [5, 64, 777, 3001])
def test_views(C, x, y):
    place = Apart()
    t, dy = place.inside(rows(45, C, x, 12)), place.inside(draw((45, C), y, 13))
    w, bias = (place.inside(v[None])[0] for v in weights(C, 14))
    out, dx = place.out(45, C, DT[y]), place.out(45, C, DT[y])
    dw, db = place.out(1, C, torch.float32)[0], place.out(1, C, torch.float32)[0]
    b.layer_norm_fwd(t, w, bias, out, eps=EPS)
    close("y", out, *layer_norm(t, w, bias, EPS, DT[y]))
    run_bwd(t, w, dy, dx, dw, db)
    for name, got, want in zip(("dx", "dw", "db"), (dx, dw, db), layer_norm_grad(t, w, dy, EPS)):
        close(name, got, *want)
    place.check()
    # a gradient that is one row for all
    same = draw((1, C), y, 15).expand(45, C)
    run_bwd(t, w, same, dx, dw, db)
    for name, got, want in zip(("dx", "dw", "db"), (dx, dw, db), layer_norm_grad(t, w, same, EPS)):
        close(name, got, *want)


def test_large_offsets_keep_their_digits():
    """A mean a thousand times the deviation: the variance is a mean of squared deviations."""
    x = 1000 + draw((30, 2000), "f32", 16)
    out = new(30, 2000, "f32")
    b.layer_norm_fwd(x, None, None, out, eps=0.0)
    close("y", out, *layer_norm(x, None, None, 0.0, torch.float32))


def test_rows_without_variance():
    x = torch.zeros((4, 100), device=DEV)
    x[1], x[2] = 3.0, -2.0 ** 40
    out = new(4, 100, "f32")
    b.layer_norm_fwd(x, None, torch.arange(100.0, device=DEV), out)
    assert torch.equal(out, torch.arange(100.0, device=DEV).expand(4, 100))
    dx = new(4, 100, "f32")
    dy = draw((4, 100), "f32", 17)
    run_bwd(x, None, dy, dx, None, None)
    close("dx", dx, *layer_norm_grad(x, None, dy, EPS)[0])


def test_a_bad_row_stays_alone():
    x, dy = rows(50, 300, "f32", 18), draw((50, 300), "f32", 19)
    x[7, 3], x[20, 0] = float("nan"), float("inf")
    out, dx = new(50, 300, "f32"), new(50, 300, "f32")
    b.layer_norm_fwd(x, None, None, out)
    run_bwd(x, None, dy, dx, None, None)
    good = [i for i in range(50) if i not in (7, 20)]
    assert out[7].isnan().all() and out[20].isnan().all() and dx[7].isnan().all() and dx[20].isnan().all()
    close("y", out[good], *layer_norm(x[good], None, None, EPS, torch.float32))
    close("dx", dx[good], *layer_norm_grad(x[good], None, dy[good], EPS)[0])


def test_no_rows():
    x = torch.empty((0, 10), device=DEV)
    b.layer_norm_fwd(x, None, None, torch.empty_like(x))
    dw, db = (torch.full((10,), 2.0, device=DEV) for _ in range(2))
    run_bwd(x, None, x, None, dw, db, accumulate=True)
    assert (dw == 2).all() and (db == 2).all()
    run_bwd(x, None, x, torch.empty_like(x), dw, db)
    assert (dw == 0).all() and (db == 0).all()


@pytest.mark.parametrize("M,C", [(40000, 64), (3000, 1024)])
def test_reruns_give_the_same_bits(M, C):
    t, dy = rows(M, C, "bf16", 20), draw((M, C), "bf16", 21)
    runs = []
    for _ in range(2):
        out = [new(M, C, "bf16"), new(1, C, "f32")[0], new(1, C, "f32")[0]]
        run_bwd(t, None, dy, *out)
        runs.append(out)
    assert all(torch.equal(a, c) for a, c in zip(*runs))
    for name, got, want in zip(("dx", "dw", "db"), runs[0], layer_norm_grad(t, None, dy, EPS)):
        close(name, got, *want)


def test_gradients_against_differences():
    """Of sum(y G) in 64 bits, by central differences: off by h^2 = 1e-10 times a third derivative, which for rows whose
    deviation is about 1 is below 100, and by 2^-53 of the sum over h."""
    x, g, w = draw((3, 7), "f32", 23), draw((3, 7), "f32", 24), weights(7, 25)[0]
    bias = weights(7, 26)[1]
    dx, dw, db = new(3, 7, "f32"), new(1, 7, "f32")[0], new(1, 7, "f32")[0]
    run_bwd(x, w, g, dx, dw, db)
    want = layer_norm_grad(x, w, g, EPS)
    f = lambda x, w, bias: float((layer_norm(x, w, bias, EPS, torch.float32)[0] * g.double()).sum())
    h = 1e-5
    args = [x.double(), w.double(), bias.double()]
    for k, (got, (_, bound)) in enumerate(zip((dx, dw, db), want)):
        for i in range(got.numel()):
            ends = []
            for s in (h, -h):
                moved = [a.clone() for a in args]
                moved[k].view(-1)[i] += s
                ends.append(f(*moved))
            assert abs((ends[0] - ends[1]) / (2 * h) - float(got.flatten()[i])) < 1e-8 + 1.05 * float(bound.flatten()[i]), (k, i)


def test_past_2_31_values():
    M, C = 140000, 16384
    x = torch.zeros((M, C), dtype=torch.bfloat16, device=DEV)
    x[-3:] = draw((3, C), "bf16", 22)
    out = torch.empty_like(x)
    b.layer_norm_fwd(x, None, None, out)
    close("y", out[-3:], *layer_norm(x[-3:], None, None, EPS, torch.bfloat16))
    assert not out[:-3].any()
    run_bwd(x, None, x, out, None, None)
    close("dx", out[-3:], *layer_norm_grad(x[-3:], None, x[-3:], EPS)[0])

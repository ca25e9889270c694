"""mt_embedding_fwd and mt_embedding_bwd against the formulas; the bounds are derived in language_reference.py."""
import pytest
import torch

from language_reference import DEV, DT, Apart, close, draw, embedding, embedding_grad, integers

pytestmark = pytest.mark.gpu

from paper_2602_00125_amd import binding as b  # noqa: E402  (a missing library fails the module)


def tokens(shape, V, kind, seed=0):
    """Tokens of V rows: even, of a few rows only, of one row, or with padding on both sides of the range."""
    if kind == "one":
        return torch.full(shape, V - 1, dtype=torch.int32, device=DEV)
    ids = integers(shape, 0, max(1, V // 50) if kind == "few" else V, seed)
    if kind == "padded":
        what = integers(shape, 0, 6, seed + 1)
        ids = torch.where(what == 0, -1, torch.where(what == 1, V, torch.where(what == 2, 2 ** 31 - 1, ids))).int()
    return ids


def workspace(ids, dy, dt):
    return torch.empty(b.embedding_bwd_workspace(ids, dy, dt), dtype=torch.uint8, device=DEV)


def run_bwd(ids, dy, dt, scale=1.0, accumulate=False):
    ws = workspace(ids, dy, dt)
    ws.fill_(0xff)
    b.embedding_bwd(ids, dy, dt, scale=scale, accumulate=accumulate, workspace=ws)
    return dt


TYPES = [("f32", "f32"), ("bf16", "bf16"), ("f32", "bf16"), ("bf16", "f32")]


@pytest.mark.parametrize("t,y", TYPES)
@pytest.mark.parametrize("M,V,D", [(1, 1, 1), (1, 7, 4096), (64, 1001, 4096), (37, 50, 777), (300, 17, 8), (5, 33, 3),
                                   (1000, 4000, 100), (3, 9, 8191)])
def test_lookup(M, V, D, t, y):
    table, ids = draw((V, D), t, 1), tokens((M,), V, "padded", 2)
    out = torch.full((M, D), float("nan"), dtype=DT[y], device=DEV)
    b.embedding_fwd(ids, table, out, scale=5.656854)
    want = embedding(ids, table, torch.tensor(5.656854, device=DEV), DT[y])
    assert torch.equal(out, want)


@pytest.mark.parametrize("t,y", TYPES)
def test_lookup_of_views(t, y):
    place = Apart()
    ids = tokens((9, 14), 40, "padded", 3)
    table = place.inside(draw((40, 77), t, 4))
    for view in (ids, ids.T, ids[:, 1:9], ids[::2, ::3], ids[:, 5], ids[:1].expand(6, 14)):
        out = place.out(view.numel(), 77, DT[y])
        b.embedding_fwd(view, table, out, scale=-0.5)
        assert torch.equal(out, embedding(view, table, -0.5, DT[y]))
    place.check()


@pytest.mark.parametrize("y", ["f32", "bf16"])
@pytest.mark.parametrize("kind", ["even", "few", "one", "padded"])
@pytest.mark.parametrize("M,V,D", [(1, 1, 1), (16, 1, 8), (17, 5, 33), (1000, 300, 77), (5000, 70000, 24), (4096, 513, 256),
                                   (2500, 20, 1030), (33, 100000, 5), (2048, 700, 500),
                                   (2049, 700, 40), (300, 17000, 4100)])
def test_gradient(M, V, D, kind, y):
    ids, dy = tokens((M,), V, kind, 5), draw((M, D), y, 6)
    if kind == "padded":  # rows without a token may hold anything
        dy[(ids < 0) | (ids >= V)] = float("nan")
    dt = torch.full((V, D), float("nan"), device=DEV)
    run_bwd(ids, dy, dt, 3.0)
    close("dtable", dt, *embedding_grad(ids, dy, V, 3.0))
    again = torch.full_like(dt, 9.0)
    assert torch.equal(run_bwd(ids, dy, again, 3.0), dt)


@pytest.mark.parametrize("y", ["f32", "bf16"])
@pytest.mark.parametrize("kind", ["even", "one", "padded"])
def test_gradient_is_added(kind, y):
    ids, dy, old = tokens((6, 171), 90, kind, 7), draw((6 * 171, 45), y, 8), draw((90, 45), "f32", 9)
    dt = run_bwd(ids, dy, old.clone(), -0.25, accumulate=True)
    close("dtable", dt, *embedding_grad(ids, dy, 90, -0.25, old))
    alone = torch.bincount(ids.flatten()[(ids.flatten() >= 0) & (ids.flatten() < 90)].long(), minlength=90) == 0
    assert torch.equal(dt[alone], old[alone])


@pytest.mark.parametrize("y", ["f32", "bf16"])
def test_gradient_of_views(y):
    place = Apart()
    ids = tokens((12, 40), 25, "padded", 10)
    ids = torch.cat([ids, tokens((60, 40), 25, "padded", 18)])  # many tokens, and below a few
    for view in (ids, ids.T, ids[::2, 1::3], ids[:12], ids[:12].T):
        dy = place.inside(draw((view.numel(), 21), y, 11))
        dt = place.out(25, 21, torch.float32)
        run_bwd(view, dy, dt)
        close("dtable", dt, *embedding_grad(view, dy, 25, 1.0))
    place.check()
    # one row for all tokens
    ids = tokens((300,), 25, "even", 12)
    dy = draw((1, 21), y, 13).expand(300, 21)
    dt = torch.empty((25, 21), device=DEV)
    run_bwd(ids, dy, dt)
    close("dtable", dt, *embedding_grad(ids, dy, 25, 1.0))


def test_runs_that_end_at_every_place():
    """Runs of all lengths, so that they begin, end and go on at every place of a chunk."""
    n = torch.arange(1, 120)
    ids = torch.repeat_interleave(torch.arange(119), n).int().to(DEV)
    ids = ids[torch.randperm(len(ids), generator=torch.Generator("cpu").manual_seed(1)).to(DEV)]
    dy = draw((len(ids), 300), "f32", 14)
    dt = torch.empty((119, 300), device=DEV)
    run_bwd(ids, dy, dt)
    close("dtable", dt, *embedding_grad(ids, dy, 119, 1.0))


@pytest.mark.parametrize("M", [2000, 5000])
def test_few_and_many_tokens_keep_apart(M):
    """Rows between those that tokens name stay as they are, or become 0, at every place of a range of rows."""
    V = 40000
    ids = torch.randperm(V, generator=torch.Generator("cpu").manual_seed(M))[:M].int().to(DEV)
    dy, old = draw((M, 12), "f32", 19), draw((V, 12), "f32", 20)
    dt = run_bwd(ids, dy, old.clone(), accumulate=True)
    want = old.clone()
    want[ids.long()] += dy
    assert torch.equal(dt, want)
    run_bwd(ids, dy, dt.fill_(float("nan")))
    assert torch.equal(dt, torch.zeros_like(dt).index_copy_(0, ids.long(), dy))


def test_the_order_of_a_token_s_rows_is_theirs():
    """Sums are taken in the tokens' order: one of values that cancel has one answer, wherever other tokens stand."""
    a, s = 2.0 ** 30, 1.0
    dy = torch.tensor([a, s, -a, s], device=DEV)[:, None].repeat(1, 9)
    want = torch.tensor(1.0)
    for V, first in ((3, 0), (70000, 65000)):
        ids = torch.full((14,), -1, dtype=torch.int32, device=DEV)
        ids[[1, 5, 6, 13]] = first + 1
        rows = torch.zeros((14, 9), device=DEV)
        rows[[1, 5, 6, 13]] = dy
        dt = torch.empty((V, 9), device=DEV)
        run_bwd(ids, rows, dt)
        assert (dt[first + 1].cpu() == want).all()


@pytest.mark.parametrize("M,V,D", [(50, 30, 21), (3000, 400, 70)])
def test_gradient_is_the_lookup_s_adjoint(M, V, D):
    """<dy, lookup(H)> = <gradient(dy), H> for every H; of small whole numbers both are exact."""
    ids = tokens((M,), V, "padded", 21)
    H, dy = (integers(s, -8, 9, 22 + i).float() for i, s in enumerate(((V, D), (M, D))))
    out, dt = torch.empty((M, D), device=DEV), torch.empty((V, D), device=DEV)
    b.embedding_fwd(ids, H, out, scale=2.0)
    run_bwd(ids, dy, dt, 2.0)
    assert (out.double() * dy.double()).sum() == (dt.double() * H.double()).sum() != 0


def test_nothing_to_look_up():
    table = draw((5, 6), "f32", 15)
    none = torch.empty((0,), dtype=torch.int32, device=DEV)
    b.embedding_fwd(none, table, torch.empty((0, 6), device=DEV))
    dt = torch.full((5, 6), 3.0, device=DEV)
    run_bwd(none, torch.empty((0, 6), device=DEV), dt, accumulate=True)
    assert (dt == 3).all()
    run_bwd(none, torch.empty((0, 6), device=DEV), dt)
    assert (dt == 0).all()
    ids = torch.full((40,), -1, dtype=torch.int32, device=DEV)
    dt.fill_(float("nan"))
    run_bwd(ids, torch.full((40, 6), float("nan"), device=DEV), dt)
    assert (dt == 0).all()
    b.embedding_fwd(ids[:3], torch.empty((0, 6), device=DEV), out := torch.full((3, 6), 2.0, device=DEV))
    assert (out == 0).all()


def test_tables_past_2_31_values():
    V, D = (1 << 21) + 3, 1024
    table = torch.zeros((V, D), dtype=torch.bfloat16, device=DEV)
    table[V - 1] = draw((D,), "bf16", 16)
    ids = torch.tensor([V - 1, 0, V - 1, V], dtype=torch.int32, device=DEV)
    out = torch.empty((4, D), dtype=torch.bfloat16, device=DEV)
    b.embedding_fwd(ids, table, out)
    assert torch.equal(out, embedding(ids, table, 1.0, torch.bfloat16))
    del table
    dt = torch.full((V, D), float("nan"), device=DEV)
    dy = draw((4, D), "f32", 17)
    run_bwd(ids, dy, dt)
    assert torch.equal(dt[V - 1], dy[0] + dy[2]) and torch.equal(dt[0], dy[1])
    assert not dt[1:V - 1].any()

"""mt_embedding_bwd's sums of an id that many tokens share. A chunk of up to 64 rows is added in fp32, U = 2^-24 an
addition (a longer one, of more values than 2^36, in 64 bits and rounded); the chunks in 64 bits, which leaves the sum's
own rounding and that of its product with the scale. So a sum is off by (64 + 2) U of its absolute terms however many
tokens there are."""
import pytest
import torch

from language_reference import DEV, DT, U, close

pytestmark = pytest.mark.gpu

from paper_2602_00125_amd import binding as b  # noqa: E402  (a missing library fails the module)


@pytest.mark.parametrize("y", ["f32", "bf16"])
@pytest.mark.parametrize("M,D", [(1 << 20, 256), (1 << 20, 1030), (3_000_001, 64), (5_000_000, 3), (1 << 24, 260), (1 << 26, 16384)])
def test_an_id_of_many_tokens(M, D, y):
    """All rows alike, so that the additions' roundings have one sign; every third column another value."""
    dy = torch.full((1, D), 0.1, device=DEV).to(DT[y])
    dy[:, ::3] = 1.7
    ids = torch.full((M,), 1, dtype=torch.int32, device=DEV)
    ids[5], ids[M // 2] = 0, 2
    dt = torch.full((3, D), float("nan"), device=DEV)
    ws = torch.full((b.embedding_bwd_workspace(ids, dy.expand(M, D), dt),), 0xff, dtype=torch.uint8, device=DEV)
    b.embedding_bwd(ids, dy.expand(M, D), dt, scale=3.0, workspace=ws)
    want = 3 * dy.double() * torch.tensor([[1], [M - 2], [1]], device=DEV)
    close("dtable", dt, want, (64 + 2) * U * want)
    old = torch.full((3, D), 2.5, device=DEV)
    b.embedding_bwd(ids, dy.expand(M, D), old, scale=3.0, accumulate=True, workspace=ws)
    close("added", old, want + 2.5, (64 + 2) * U * want + U * (want + 2.5))


@pytest.mark.parametrize("M,D", [(1 << 20, 300), (2_000_003, 12)])
def test_no_token_is_lost(M, D):
    """Of small whole numbers all sums are exact."""
    g = torch.Generator(DEV)
    g.manual_seed(1)
    dy = torch.randint(-3, 4, (M, D), generator=g, device=DEV).float()
    ids = torch.randint(-1, 5, (M,), generator=g, device=DEV, dtype=torch.int32)
    dt = torch.full((4, D), float("nan"), device=DEV)
    ws = torch.full((b.embedding_bwd_workspace(ids, dy, dt),), 0xff, dtype=torch.uint8, device=DEV)
    b.embedding_bwd(ids, dy, dt, workspace=ws)
    for v in range(4):
        assert torch.equal(dt[v].double(), dy[ids == v].double().sum(0)), v

"""mt_layer_norm_bwd's sums over rows, dw and db, where a lane meets several rows: no row is lost and none counts twice,
and their rounding does not grow with the rows.

A lane adds its rows one after another, 128 of them at most, in fp32 (U = 2^-24 an addition); what the lanes and blocks
have is added in 64 bits, a block's part and the result are rounded once each. So db is off by (n + 3) U sum|dy| for n
rows a lane, and dw besides by what n_i is off by (language_reference.py). Sums of small whole numbers are exact.
"""
import pytest
import torch

from language_reference import DEV, DT, U, _standard, close, draw, integers

pytestmark = pytest.mark.gpu

from paper_2602_00125_amd import binding as b  # noqa: E402  (a missing library fails the module)

EPS = 1e-5


def run(x, w, dy, dw, db, accumulate=False):
    ws = torch.full((b.layer_norm_bwd_workspace(x, w, dy, None, dw, db),), 0xff, dtype=torch.uint8, device=DEV)
    b.layer_norm_bwd(x, w, dy, None, dw, db, eps=EPS, accumulate=accumulate, workspace=ws)


# rows of a wave's part, of a wave, of several; more than one pass of all blocks holds
SIZES = [(300000, 7), (40000, 64), (40000, 100), (9001, 777), (9001, 1024), (2500, 2560), (1300, 8192), (1111, 7001), (700, 16384)]


@pytest.mark.parametrize("x,y", [("f32", "f32"), ("bf16", "bf16"), ("f32", "bf16"), ("bf16", "f32")])
@pytest.mark.parametrize("M,C", SIZES)
def test_no_row_is_lost(M, C, x, y):
    t, dy = draw((M, C), x, 1), integers((M, C), -3, 4, 2).to(DT[y])
    w = 1 + 0.2 * draw((C,), "f32", 3)
    dw, db = (torch.full((C,), float("nan"), device=DEV) for _ in range(2))
    run(t, w, dy, dw, db)
    assert torch.equal(db.double(), dy.double().sum(0))
    n, _, en, _ = _standard(t, EPS)
    terms = dy.double() * n
    want, bound = terms.sum(0), (dy.double().abs() * en).sum(0) + (8 + 3) * U * terms.abs().sum(0)
    close("dw", dw, want, bound)
    old = [integers((C,), -9, 10, 4).float(), draw((C,), "f32", 5)]
    both = [old[1].clone(), old[0].clone()]
    run(t, w, dy, *both, accumulate=True)
    assert torch.equal(both[1].double(), dy.double().sum(0) + old[0].double())
    close("dw", both[0], want + old[1].double(), bound + U * (want + old[1].double()).abs())


@pytest.mark.parametrize("x,y", [("f32", "f32"), ("bf16", "bf16")])
@pytest.mark.parametrize("M,C", [(1 << 20, 4104), (1 << 20, 4101), (1 << 22, 777), (1 << 23, 64), (5_000_000, 4101)])
def test_many_rows_of_one_sign(M, C, x, y):
    """One row for all: sums of equal terms, whose roundings all have one sign."""
    t, dy = draw((1, C), x, 6).expand(M, C), torch.full((1, C), 0.1, device=DEV).to(DT[y])
    dy[:, ::3] = 1.1
    dw, db = (torch.full((C,), float("nan"), device=DEV) for _ in range(2))
    run(t, None, dy.expand(M, C), dw, db)
    want = M * dy[0].double()
    close("db", db, want, (128 + 3) * U * want)
    n, _, en, _ = _standard(t[:1], EPS)
    close("dw", dw, want * n[0], want * en[0] + (128 + 3) * U * (want * n[0]).abs())

"""mt_dropout_fwd and mt_dropout_bwd: the mask bit by bit against the generator written out in Python's integers,
the values against 64 bits."""
import math

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

from paper_2602_00125_amd import binding as b  # noqa: E402  (a missing library fails the module)

DEV = "cuda:0"
DT = {"f32": torch.float32, "bf16": torch.bfloat16}
SEED, OFFSET = 0x9ABCDEF012345678, (1 << 32) - 3  # the counter passes 32 bits after three steps


def draw(shape, dtype, seed):
    g = torch.Generator("cpu")
    g.manual_seed(seed)
    return torch.randn(shape, generator=g).to(DT[dtype]).to(DEV)


def words(counter, key):
    """Philox4x32-10 of one counter."""
    m = 0xFFFFFFFF
    x, k = [counter & m, counter >> 32 & m, 0, 0], [key & m, key >> 32]
    for _ in range(10):
        p, q = x[0] * 0xD2511F53, x[2] * 0xCD9E8D57
        x = [q >> 32 ^ x[1] ^ k[0], q & m, p >> 32 ^ x[3] ^ k[1], p & m]
        k = [k[0] + 0x9E3779B9 & m, k[1] + 0xBB67AE85 & m]
    return x


def test_generator_against_published_values():
    """Known answers of the paper's reference implementation: all-zero counter and key."""
    assert words(0, 0) == [0x6627E8D5, 0xE169C58D, 0xBC57AC4C, 0x9B00DBD8]


def stays(n, p, seed=SEED, offset=OFFSET):
    drop = round(p * 65536)
    bits = []
    for c in range((n + 7) // 8):
        for w in words((offset + c) % 2 ** 64, seed):
            bits += [w & 0xFFFF, w >> 16]
    keep = np.array(bits[:n]) >= drop
    return torch.from_numpy(keep).to(DEV), 65536 / (65536 - drop) if drop < 65536 else 0.0


def expect(x, res, keep, scale):
    y = torch.where(keep.view(x.shape), x.double() * scale, 0.0)
    return y if res is None else y + res.double()


def close(got, want, res):
    # fp32: the scale, the product and the sum are rounded; bf16: the result once more
    u = 2.0 ** -8 if got.dtype == torch.bfloat16 else 0.0
    size = want.abs() if res is None else want.abs() + 2 * res.double().abs()
    assert ((got.double() - want).abs() <= 1.01 * u * want.abs() + 2.0 ** -22 * size).all()


SHAPES = [(1, 1), (1, 7), (3, 8), (5, 13), (64, 64), (17, 1000), (509, 3), (2, 4096)]


@pytest.mark.parametrize("x,y", [("f32", "f32"), ("bf16", "bf16"), ("f32", "bf16"), ("bf16", "f32")])
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_sizes(shape, x, y):
    p = 0.3
    keep, scale = stays(shape[0] * shape[1], p)
    t, res = draw(shape, x, 0), draw(shape, y, 1)
    out = torch.full(shape, math.nan, dtype=DT[y], device=DEV)
    b.dropout_fwd(t, res, p, SEED, OFFSET, out)
    close(out, expect(t, res, keep, scale), res)
    b.dropout_fwd(t, None, p, SEED, OFFSET, out)
    close(out, expect(t, None, keep, scale), None)
    out.fill_(math.nan)
    b.dropout_bwd(t, p, SEED, OFFSET, out)
    close(out, expect(t, None, keep, scale), None)
    out.copy_(res)
    b.dropout_bwd(t, p, SEED, OFFSET, out, accumulate=True)
    close(out, expect(t, res, keep, scale), res)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("M,N,pitch,shift", [(7, 24, 32, 0), (7, 24, 27, 0), (7, 23, 40, 0), (7, 24, 24, 1),
                                             (9, 40, 64, 3)])
def test_pitches_and_bases(dtype, M, N, pitch, shift):
    """The mask follows the row-major index whatever the strides, and nothing between the rows is written."""
    keep, scale = stays(M * N, 0.5)

    def place(t):
        buf = torch.full((M * pitch + shift,), 5.0, dtype=DT[dtype], device=DEV)
        view = buf[shift:].view(M, pitch)[:, :N]
        view.copy_(t)
        return buf, view
    (_, x), (_, res), (buf, y) = (place(draw((M, N), dtype, i)) for i in range(3))
    b.dropout_fwd(x, res, 0.5, SEED, OFFSET, y)
    close(y, expect(x, res, keep, scale), res)
    gaps = buf[shift:].view(M, pitch)[:, N:]
    assert (gaps == 5.0).all() and (buf[:shift] == 5.0).all()


@pytest.mark.parametrize("p", [0.0, 1e-6, 1 / 65536, 0.1, 0.999995, 1.0])
def test_probabilities(p):
    x, res = draw((11, 40), "f32", 0), draw((11, 40), "f32", 1)
    keep, scale = stays(440, np.float32(p).item())
    y = torch.full_like(x, math.nan)
    b.dropout_fwd(x, res, p, SEED, OFFSET, y)
    close(y, expect(x, res, keep, scale), res)
    if p == 0.0:
        b.dropout_fwd(x, None, p, SEED, OFFSET, y)
        assert torch.equal(y, x)


def test_a_dropped_infinity_is_zero():
    x = torch.full((4, 64), math.inf, device=DEV)
    x[1] = math.nan
    keep, _ = stays(256, 0.5)
    y = torch.empty_like(x)
    b.dropout_fwd(x, None, 0.5, SEED, OFFSET, y)
    assert (y[~keep.view(4, 64)] == 0).all() and not y[keep.view(4, 64)].isfinite().any()


def test_share_kept_and_calls_that_follow_one_another():
    """A million elements: the share kept within five deviations of p; the second half of a call is a call of its
    own from the counters after the first half's."""
    M, N, p = 1024, 1024, 0.1
    x, y, z = torch.ones(M, N, device=DEV), torch.empty(M, N, device=DEV), torch.empty(M // 2, N, device=DEV)
    b.dropout_fwd(x, None, p, 5, 100, y)
    share = (y != 0).double().mean().item()
    assert abs(share - 0.9) < 5 * math.sqrt(0.09 / (M * N)) + 2.0 ** -16
    b.dropout_fwd(x[M // 2:], None, p, 5, 100 + M * N // 16, z)
    assert torch.equal(z, y[M // 2:])
    other = torch.empty_like(y)
    b.dropout_fwd(x, None, p, 6, 100, other)
    assert 0.15 < ((y != 0) != (other != 0)).double().mean().item() < 0.21  # 2 * 0.1 * 0.9


def test_replays_from_a_graph():
    x, res, y = draw((33, 100), "bf16", 0), draw((33, 100), "bf16", 1), torch.empty(33, 100, dtype=torch.bfloat16, device=DEV)
    call = lambda: b.dropout_fwd(x, res, 0.2, SEED, OFFSET, y)
    call()
    want = y.clone()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        call()
    torch.cuda.current_stream().wait_stream(side)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        call()
    for _ in range(3):
        y.fill_(math.nan)
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, want)
        call()
        torch.cuda.synchronize()
        assert torch.equal(y, want)


def test_indices_past_32_bits():
    N, tail, p = (1 << 32) + 4099, 9000, 0.4  # elements; bf16: 8.6 GB
    at = (N - tail) // 8 * 8
    x = torch.empty((1, N), dtype=torch.bfloat16, device=DEV)
    y = torch.empty_like(x)
    x[:, at:].copy_(torch.randn((1, N - at), generator=torch.Generator("cpu").manual_seed(1)))
    b.dropout_fwd(x, None, p, 9, 3, y)
    part = torch.empty((1, N - at), dtype=torch.bfloat16, device=DEV)
    b.dropout_fwd(x[:, at:], None, p, 9, 3 + at // 8, part)
    torch.cuda.synchronize()
    assert torch.equal(y[:, at:], part)

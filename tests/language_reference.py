"""The embedding, layer norm, cross-entropy and gradient clipping, and how far fp32 / bf16 kernels may be from them, in
64 bits.

The bounds are first order in the roundings the kernels make, with 5% on top for the products of two errors: U = 2^-24
for an fp32 operation, half a step of the output's type for its rounding (``half``). A sum of n terms added in any order
is off by at most n U of its absolute terms; a row's sums are trees: 64 values a lane at most, 64 lanes, 16 waves, so 64 +
6 + 16 additions and, for a mean, the product with a rounded 1 / C: DEPTH.
"""
from __future__ import annotations

import torch

U = 2.0 ** -24
DEPTH = 90
ABS = 2.0 ** -126  # denormals may be flushed
DEV = "cuda:0"
DT = {"f32": torch.float32, "bf16": torch.bfloat16}


def half(dtype):
    return torch.finfo(dtype).eps / 2


def draw(shape, dtype="f32", seed=0, scale=1.0, shift=0.0):
    g = torch.Generator("cpu")
    g.manual_seed(seed)
    return (shift + scale * torch.randn(shape, generator=g)).to(DT[dtype]).to(DEV)


def integers(shape, lo, hi, seed=0):
    g = torch.Generator("cpu")
    g.manual_seed(seed)
    return torch.randint(lo, hi, shape, generator=g, dtype=torch.int32).to(DEV)


class Apart:
    """Matrices inside larger buffers, at odd places and pitches: ``inside(t)`` a copy of t that a kernel may read,
    ``out(shape)`` one that it writes; ``check()`` that it wrote nothing beside them."""

    def __init__(self, off=3, extra=5):
        self.off, self.extra, self.bufs = off, extra, []

    def _view(self, buf, rows, cols):
        return buf[self.off:].as_strided((rows, cols), (cols + self.extra, 1), self.off)

    def _make(self, rows, cols, dtype):
        buf = torch.full((self.off + rows * (cols + self.extra) + 16,), 7.0, dtype=dtype, device=DEV)
        return buf, self._view(buf, rows, cols)

    def inside(self, t):
        buf, v = self._make(*t.shape, t.dtype)
        buf.fill_(float("nan"))
        v.copy_(t)
        return v

    def out(self, rows, cols, dtype):
        buf, v = self._make(rows, cols, dtype)
        v.fill_(float("nan"))
        self.bufs.append((buf, v))
        return v

    def check(self):
        for buf, v in self.bufs:
            keep = torch.ones_like(buf, dtype=torch.bool)
            self._view(keep, *v.shape).fill_(False)
            assert (buf[keep] == 7).all(), "written beside the output"


def close(name, got, want, bound):
    assert got.shape == want.shape, (name, got.shape, want.shape)
    got = got.double()
    assert torch.equal(got.isfinite(), want.isfinite()), f"{name}: finite in other places"
    fin = want.isfinite()
    assert torch.equal(got[~fin].nan_to_num(1.0), want[~fin].nan_to_num(1.0)), f"{name}: infinities differ"
    err = torch.where(fin, (got - want).abs(), 0.0)
    bad = err > torch.where(fin, bound, 0.0) * 1.05 + ABS
    if bad.any():
        i = int(torch.where(bad, err / (bound + ABS), 0.0).argmax())
        raise AssertionError(f"{name}: {int(bad.sum())} of {bad.numel()} out of bounds; worst at {i}: got "
                             f"{got.flatten()[i].item()!r} want {want.flatten()[i].item()!r} bound "
                             f"{bound.expand_as(want).flatten()[i].item():.3e}")


# ------------------------------------------------------------------ embedding
def embedding(ids, table, scale, dtype):
    """y itself: a product and a rounding have one right answer."""
    i = ids.flatten().long()
    ok = (i >= 0) & (i < table.shape[0])
    rows = table[torch.where(ok, i, 0)].float() * scale
    return torch.where(ok[:, None], rows, 0.0).to(dtype)


def embedding_grad(ids, dy, V, scale, old=None):
    """dtable and its bound: the n terms of a row, their product with the scale, the addition to what was there."""
    scale = float(torch.tensor(scale, dtype=torch.float32))
    i = ids.flatten().long()
    ok = (i >= 0) & (i < V)
    i, d = i[ok], dy[ok].double()
    zeros = lambda: torch.zeros((V, dy.shape[1]), dtype=torch.float64, device=dy.device)
    g, a = zeros().index_add_(0, i, d) * scale, zeros().index_add_(0, i, d.abs()) * abs(scale)
    n = torch.bincount(i, minlength=V)[:, None]
    bound = (n + 1) * U * a
    if old is not None:
        g = g + old.double()
        bound = bound + U * (n > 0) * g.abs()
    return g, bound


# ----------------------------------------------------------------- layer norm
def _standard(x, eps):
    """n, r, and their errors: of n absolute, of r relative."""
    x = x.double()
    mean = x.mean(-1, keepdim=True)
    d = x - mean
    var = d.square().mean(-1, keepdim=True)
    r = (var + eps).rsqrt()
    n = d * r
    ed = DEPTH * U * x.abs().mean(-1, keepdim=True) + U * d.abs()
    ev = 2 * (d.abs() * ed).mean(-1, keepdim=True) + DEPTH * U * var + U * (var + eps)
    er = 0.5 * ev * r * r + 3 * U  # the root and the quotient: an ulp each
    return n, r, ed * r + n.abs() * (er + U), er


def layer_norm(x, w, b, eps, dtype):
    eps = float(torch.tensor(eps, dtype=torch.float32))
    n, _, en, _ = _standard(x, eps)
    W = 1.0 if w is None else w.double()
    B = 0.0 if b is None else b.double()
    y = n * W + B
    return y, en * abs(W) + (U + half(dtype)) * y.abs()


def layer_norm_grad(x, w, dy, eps, old=None):
    """(dx, bound), (dw, bound), (db, bound); old: what dx, dw, db held (accumulated)."""
    eps = float(torch.tensor(eps, dtype=torch.float32))
    n, r, en, er = _standard(x, eps)
    dyd = dy.double()
    g = dyd if w is None else dyd * w.double()
    mean = lambda t: t.mean(-1, keepdim=True)
    mg, mgn = mean(g), mean(g * n)
    emg = (DEPTH + 1) * U * mean(g.abs())
    emgn = mean(g.abs() * en) + (DEPTH + 3) * U * mean((g * n).abs())
    inner = g - mg - n * mgn
    size = g.abs() + mg.abs() + (n * mgn).abs()
    ein = U * g.abs() + emg + en * mgn.abs() + n.abs() * emgn + 3 * U * size
    dx = r * inner
    out = [[dx, r * ein + dx.abs() * (er + U)]]
    M = x.shape[0]
    dw = (dyd * n).sum(0)
    out.append([dw, (dyd.abs() * en).sum(0) + (M + 2) * U * (dyd * n).abs().sum(0)])
    out.append([dyd.sum(0), M * U * dyd.abs().sum(0)])
    for k, o in enumerate(out):
        if old is not None:
            o[0] = o[0] + old[k].double()
            o[1] = o[1] + U * o[0].abs()
    out[0][1] = out[0][1] + half(dy.dtype) * out[0][0].abs()
    return out


# -------------------------------------------------------------- cross-entropy
def cross_entropy(logits, targets, dtype):
    """(loss, bound), (losses, bound), (dlogits, bound)."""
    M, V = logits.shape
    t = targets.flatten().long()
    ok = (t >= 0) & (t < V)
    n = max(1, int(ok.sum()))
    z = torch.where(ok[:, None], logits.double(), 0.0)
    at = torch.where(ok, t, 0)[:, None]
    top = z.amax(-1, keepdim=True)
    # relative to the top: z - lse in 64 bits would lose lse's digits next to logits of 1e38
    e = torch.exp(z - top)
    log_sum = e.sum(-1, keepdim=True).log()
    losses = torch.where(ok, (top - z.gather(1, at) + log_sum)[:, 0], 0.0)
    p = e / e.sum(-1, keepdim=True)
    # an exponential's relative error: its argument's rounding, and 4 U of the function's and of the product with log2 e
    ee = U * torch.where(z.isinf(), 0.0, (top - z).abs()) + 4 * U
    es = (p * ee).sum(-1) + DEPTH * U  # the sum's, relative
    el = es + U * ((top - z.gather(1, at))[:, 0].abs() + 2 * log_sum[:, 0].abs() + losses.abs())
    el = torch.where(ok, el, 0.0)
    onehot = torch.zeros_like(p).scatter_(1, at, 1.0)
    d = torch.where(ok[:, None], (p - onehot) / n, 0.0)
    ed = (p * (ee + es[:, None] + 4 * U) + 2 * U * onehot) / n + (U + half(dtype)) * d.abs()
    loss = losses.sum().view(1) / n
    return [(loss, (el.sum() / n + (M + 2) * U * loss).view(1)), (losses, el), (d, torch.where(ok[:, None], ed, 0.0))]


# ------------------------------------------------------------------- clipping
def clip(grads, max_norm, out_dtypes):
    """(norm, bound) and [(out, bound)]; squares and their sum in 64 bits are exact to 1e-12."""
    norm = sum((g.double().square().sum() for g in grads), torch.zeros((), dtype=torch.float64, device=DEV)).sqrt()
    f = min(1.0, max_norm / float(norm)) if float(norm) > 0 else 1.0
    outs = []
    for g, dt in zip(grads, out_dtypes):
        y = g.double() * f
        # by way of fp32 where the result is bf16
        outs.append((y, ((U if f < 1 else 0.0) + (half(dt) if f < 1 or dt != g.dtype else 0.0) + 1e-12) * y.abs()))
    return (norm.view(1), (U + 1e-12) * norm.view(1)), outs

"""Attention, its gradients and how far fp32 / bf16 kernels may be from them, in 64 bits.

The error bounds are first order in the roundings the kernels make (u = 2^-8 for
a rounding to bf16; fp32 arithmetic counts as 1e-4 of the absolute terms, the
project's bar for fp32 sums), with 5% on top for the products of two errors:
  o:  P and o are rounded:                     (u + u) sum_j P_j |v_j|
  dv: P and dv are rounded:                    (u + u) sum_i P_i |do_i|
  dS: itself rounded, delta from a rounded o:  u |dS| + u P sum_d |do o|
  dq, dk: dS's error times |k|, |q|, and their own rounding
"""
from __future__ import annotations

import torch

ABS = 1e-6


def visible(B, TQ, TK, causal, kv_len, q_start, dev):
    j = torch.arange(TK, device=dev)
    n = torch.full((B,), TK, device=dev) if kv_len is None else kv_len.clamp(0, TK)
    seen = (j[None, None] < n[:, None, None]).expand(B, TQ, TK)
    if causal:
        start = torch.full((B,), TK - TQ, device=dev) if q_start is None else q_start
        i = torch.arange(TQ, device=dev)
        seen = seen & (j[None, None] <= start[:, None, None] + i[None, :, None])
    return seen


def reference(q, k, v, scale, causal=False, kv_len=None, q_start=None, dout=None):
    """dict of name -> (value, bound): o, lse and, with dout, dq, dk, dv (fp64, on q's device)."""
    B, TQ, HQ, D = q.shape
    TK, HK = k.shape[1:3]
    G = HQ // HK if HK else 1
    bf = q.dtype == torch.bfloat16
    u = 2.0 ** -8 if bf else 0.0
    f = 1e-5 if bf else 1e-4  # fp32 sums of exact bf16 products are closer than those of fp32 values
    seen = visible(B, TQ, TK, causal, kv_len, q_start, q.device)[:, None]
    # garbage at keys past kv_len takes no part
    exists = seen.any(2)[:, 0] if kv_len is None else torch.arange(TK, device=q.device)[None] < kv_len[:, None]
    clean = lambda x: torch.where(exists[:, :, None, None], x.double(), 0.0) if kv_len is not None else x.double()
    Q = q.double().permute(0, 2, 1, 3)
    K, V = (clean(x).permute(0, 2, 1, 3).repeat_interleave(G, 1) for x in (k, v))
    S = (Q @ K.transpose(-1, -2)) * scale
    Z = torch.where(seen, S, -torch.inf)
    if TK:
        lse = torch.logsumexp(Z, -1)
    else:
        lse = torch.full((B, HQ, TQ), -torch.inf, dtype=torch.float64, device=q.device)
    P = torch.where(seen, torch.exp(S - torch.where(lse.isinf(), 0.0, lse)[..., None]), 0.0)
    o = P @ V
    Sa = (Q.abs() @ K.abs().transpose(-1, -2)) * scale
    # an absolute error of the scores is a relative one of P (1e-6 covers sums of D <= 128 fp32 terms)
    e = 1e-6 * torch.where(seen, Sa, 0.0).amax(-1, keepdim=True) if TK else torch.zeros_like(o[..., :1])
    back = lambda x: x.permute(0, 2, 1, 3)
    out = {"o": (back(o), back(1.05 * (2 * u + f + 2 * e) * (P @ V.abs()) + ABS)),
           "lse": (lse, (f * (1 + lse.abs()) + e[..., 0]).nan_to_num(0, 0, 0))}
    if dout is None:
        return out
    dO = dout.double().permute(0, 2, 1, 3)
    dP = dO @ V.transpose(-1, -2)
    delta = (dO * o).sum(-1, keepdim=True)
    dS = P * (dP - delta)
    A = (dO * o).abs().sum(-1, keepdim=True)
    eS = (u + f + 2 * e) * dS.abs() + P * (u * A + (f + 2 * e) * (dO.abs() @ V.abs().transpose(-1, -2) + A))
    fold = lambda x: x.unflatten(1, (HK, G)).sum(2) if HK else x[:, :0]

    def entry(val, err):
        return back(val), back(1.05 * (err + u * val.abs()) + ABS)

    out["dq"] = entry(dS @ K * scale, eS @ K.abs() * scale)
    out["dk"] = entry(fold(dS.transpose(-1, -2) @ Q) * scale, fold(eS.transpose(-1, -2) @ Q.abs()) * scale)
    out["dv"] = entry(fold(P.transpose(-1, -2) @ dO), fold(((u + f + 2 * e) * P).transpose(-1, -2) @ dO.abs()))
    return out


def check(name, got, want, bound):
    got = got.double()
    assert got.shape == want.shape, (name, got.shape, want.shape)
    inf = want.isinf()
    assert torch.equal(got[inf], want[inf]), f"{name}: infinities differ"
    err = torch.where(inf, 0.0, (got - want).abs())
    assert not err.isnan().any(), f"{name}: NaN in the result"
    bad = err > bound
    if bad.any():
        i = int(torch.argmax(torch.where(bad, err / bound, 0.0)))
        raise AssertionError(f"{name}: {int(bad.sum())} of {bad.numel()} out of bounds; worst got "
                             f"{got.flatten()[i].item()!r} want {want.flatten()[i].item()!r} bound "
                             f"{bound.expand_as(want).flatten()[i].item():.3e}")

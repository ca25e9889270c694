"""An attention block trained and served with the library's operators alone.

    h = x + dropout(attention(rotate(norm(q)), rotate(norm(k)), v) Wo^T + bo),   [q k v] = x Wqkv^T + bqkv

with grouped key heads and causal attention over ragged sequences. ``AttentionBlock`` holds the parameters, every
buffer and workspace of a training step; ``step`` runs forward, mean squared error, backward and Adam, ``decode`` one
token of each sequence against a cache. fp32 throughout, or with bf16 products and attention (fp32 parameters, residual
stream and statistics): the projections' bf16 copies are made anew by every ``forward`` and after every update, and by
``refresh`` for a program that changes the parameters by itself and goes on with ``decode``.

    python examples/attention_block.py [--dtype bf16] [--steps 20] [--batch 4] [--tokens 1024] ...
"""
from __future__ import annotations

import argparse
import os
import sys
import time

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import torch

from paper_2602_00125_amd import binding as mt

DEV = "cuda:0"
EPS = 1e-6


def rotary_tables(positions: torch.Tensor, width: int, base: float = 10000.0):
    """cos and sin [..., width / 2] of the angles position base^(-2 i / width)."""
    freq = base ** (-torch.arange(0, width, 2, device=positions.device, dtype=torch.float64) / width)
    a = positions.double()[..., None] * freq
    return a.cos().float(), a.sin().float()


def _workspace(n: int):
    return torch.empty(n, dtype=torch.uint8, device=DEV) if n else None


class AttentionBlock:
    def __init__(self, batch, tokens, width, heads, kv_heads, head_width, dtype=torch.float32, p=0.1, lr=1e-3, seed=0):
        B, T, C, HQ, HK, D = batch, tokens, width, heads, kv_heads, head_width
        self.B, self.T, self.C, self.HQ, self.HK, self.D = B, T, C, HQ, HK, D
        self.dtype, self.p, self.lr, self.seed, self.t = dtype, p, lr, seed, 0
        W = (HQ + 2 * HK) * D
        g = torch.Generator(DEV)
        g.manual_seed(seed)

        def uniform(rows, cols):
            return (2 * torch.rand(rows, cols, generator=g, device=DEV) - 1) / cols ** 0.5

        f32 = dict(device=DEV, dtype=torch.float32)
        self.params = {"wqkv": uniform(W, C), "bqkv": torch.zeros(W, **f32), "gq": torch.ones(D, **f32),
                       "gk": torch.ones(D, **f32), "wo": uniform(C, HQ * D), "bo": torch.zeros(C, **f32)}
        zeros = lambda: {n: torch.zeros_like(t) for n, t in self.params.items()}
        self.grads, self.m, self.v = zeros(), zeros(), zeros()
        self.cos, self.sin = (t.expand(B, T, -1) for t in rotary_tables(torch.arange(T, device=DEV)[None], D))
        # activations and their gradients, in the products' type or in fp32
        act = dict(device=DEV, dtype=dtype)
        M = B * T
        self.qkv, self.y, self.h = (torch.empty(M, n, **f32) for n in (W, C, C))
        self.q, self.k, self.vv = (torch.empty(B, T, n, D, **act) for n in (HQ, HK, HK))
        self.o, self.lse = torch.empty(B, T, HQ, D, **act), torch.empty(B, HQ, T, **f32)
        self.dh, self.dx = torch.empty(M, C, **f32), torch.empty(M, C, **f32)
        self.dy, self.dqkv = torch.empty(M, C, **act), torch.empty(M, W, **act)
        self.do32 = torch.empty(M, HQ * D, **f32)
        self.do = torch.empty(B, T, HQ, D, **act)
        self.dq, self.dk = torch.empty_like(self.q), torch.empty_like(self.k)
        self.loss = torch.empty(1, **f32)
        self.x16, self.w16 = None, {}
        if dtype != torch.float32:
            self.x16 = torch.empty(M, C, **act)
            self.w16 = {n: torch.empty_like(self.params[n], dtype=dtype) for n in ("wqkv", "wo")}
        self.refresh()
        kw = dict(causal=True, kv_len=torch.zeros(B, dtype=torch.int32, device=DEV))
        q32, k32, _ = self._heads(self.qkv)
        dq, dk, dv = self._heads(self.dqkv)
        attn = (self.q, self.k, self._values(), self.o, self.lse)
        p = self.params
        self.ws = _workspace(max(
            mt.attention_fwd_workspace(*attn, **kw), mt.attention_bwd_workspace(*attn, self.do, self.dq, self.dk, dv, **kw),
            mt.qk_norm_rope_bwd_workspace(q32, k32, p["gq"], p["gk"], self.cos, self.sin, self.dq, self.dk, dq, dk,
                                          self.grads["gq"], self.grads["gk"]),
            mt.linear_bwd_workspace(self._operand("x", self.h), self._weight("wqkv"), self.dqkv, self.dx, self.grads["wqkv"],
                                    self.grads["bqkv"]),
            mt.linear_bwd_workspace(self.o.view(M, -1), self._weight("wo"), self.dy, self.do32, self.grads["wo"],
                                    self.grads["bo"]),
            mt.mse_loss_workspace(self.h, self.dh)))

    # ---------------------------------------------------------------- views and casts
    def _heads(self, packed, B=None, T=None):
        """q, k, v [B, T, heads, D]: views of a packed projection's rows."""
        B, T, HQ, HK, D = B or self.B, T or self.T, self.HQ, self.HK, self.D
        rows = packed.view(B, T, -1)
        cut = lambda a, n: rows[..., a * D:(a + n) * D].unflatten(-1, (n, D))
        return cut(0, HQ), cut(HQ, HK), cut(HQ + HK, HK)

    def _values(self):
        """The values attention reads: the projection's own in fp32, a copy in bf16."""
        return self._heads(self.qkv)[2] if self.dtype == torch.float32 else self.vv

    def _operand(self, name, t):
        return t if self.dtype == torch.float32 else self.x16

    def _weight(self, name):
        return self.params[name] if self.dtype == torch.float32 else self.w16[name]

    @staticmethod
    def _cast(src, dst):
        mt.dropout_fwd(src, None, 0.0, 0, 0, dst)  # p = 0: a copy, rounded to dst's type

    def refresh(self):
        """The bf16 copies of the projections from the parameters (nothing to do in fp32)."""
        for n, w in self.w16.items():
            self._cast(self.params[n], w)

    # ---------------------------------------------------------------------- training
    def forward(self, x, kv_len):
        """x [B T, C] fp32 -> h [B T, C]; tokens from kv_len on are padding."""
        P, M = self.params, self.B * self.T
        if self.dtype != torch.float32:
            self._cast(x, self.x16)
        self.refresh()
        mt.linear_fwd(self._operand("x", x), self._weight("wqkv"), P["bqkv"], self.qkv)
        q, k, _ = self._heads(self.qkv)
        mt.qk_norm_rope_fwd(q, k, P["gq"], P["gk"], self.cos, self.sin, self.q, self.k, eps=EPS)
        if self.dtype != torch.float32:
            self._cast(self.qkv[:, (self.HQ + self.HK) * self.D:], self.vv.view(M, -1))
        mt.attention_fwd(self.q, self.k, self._values(), self.o, self.lse, kv_len=kv_len, causal=True, workspace=self.ws)
        mt.linear_fwd(self.o.view(M, -1), self._weight("wo"), P["bo"], self.y)
        mt.dropout_fwd(self.y, x, self.p, self.seed, self._offset(), self.h)

    def _offset(self):
        return self.t * ((self.B * self.T * self.C + 7) // 8)  # a step's share of the generator's counters

    def backward(self, x, kv_len):
        """From dh: the gradients of the parameters and, in dx, of x."""
        P, G, M = self.params, self.grads, self.B * self.T
        mt.dropout_bwd(self.dh, self.p, self.seed, self._offset(), self.dy)
        o = self.o.view(M, -1)
        do32 = self.do.view(M, -1) if self.dtype == torch.float32 else self.do32
        mt.linear_bwd(o, self._weight("wo"), self.dy, do32, G["wo"], G["bo"], workspace=self.ws)
        if self.dtype != torch.float32:
            self._cast(do32, self.do.view(M, -1))
        dq, dk, dv = self._heads(self.dqkv)
        mt.attention_bwd(self.q, self.k, self._values(), self.o, self.lse, self.do, self.dq, self.dk, dv, kv_len=kv_len,
                         causal=True, workspace=self.ws)
        q, k, _ = self._heads(self.qkv)
        mt.qk_norm_rope_bwd(q, k, P["gq"], P["gk"], self.cos, self.sin, self.dq, self.dk, dq, dk, G["gq"], G["gk"], eps=EPS,
                            workspace=self.ws)
        self.dx.copy_(self.dh)  # through the residual
        mt.linear_bwd(self._operand("x", x), self._weight("wqkv"), self.dqkv, None, G["wqkv"], G["bqkv"], workspace=self.ws)
        mt.linear_bwd(None, self._weight("wqkv"), self.dqkv, self.dx, accumulate=True, workspace=self.ws)

    def step(self, x, target, kv_len):
        """One training step; the loss stays on the device (self.loss)."""
        self.forward(x, kv_len)
        mt.mse_loss(self.h, target, self.loss, self.dh, workspace=self.ws)
        self.backward(x, kv_len)
        self.t += 1
        mt.adam_step(list(self.params.values()), list(self.grads.values()), list(self.m.values()), list(self.v.values()),
                     self.lr, 0.9, 0.999, 1e-8, self.t)
        self.refresh()

    # ----------------------------------------------------------------------- serving
    def decode(self, x, k_cache, v_cache, lens):
        """One token of each sequence: x [B, C] fp32 and caches [B, tokens, HK, D] holding lens [B] int32 tokens each;
        appends the new keys and values and returns h [B, C] (no dropout). The caller counts lens up."""
        B, P = x.shape[0], self.params
        x16 = x if self.dtype == torch.float32 else x.to(self.dtype)
        qkv = torch.empty(B, self.qkv.shape[1], device=DEV)
        mt.linear_fwd(x16, self._weight("wqkv"), P["bqkv"], qkv)
        q32, k32, v32 = self._heads(qkv, B, 1)
        q, k = (torch.empty(t.shape, dtype=self.dtype, device=DEV) for t in (q32, k32))
        cos, sin = (t[:, None] for t in rotary_tables(lens, self.D))
        mt.qk_norm_rope_fwd(q32, k32, P["gq"], P["gk"], cos, sin, q, k, eps=EPS)
        row = torch.arange(B, device=DEV)
        k_cache[row, lens.long()] = k[:, 0]
        v_cache[row, lens.long()] = v32[:, 0].to(self.dtype)
        o = torch.empty_like(q)
        ws = _workspace(mt.attention_fwd_workspace(q, k_cache, v_cache, o, causal=True, kv_len=lens + 1, q_start=lens))
        mt.attention_fwd(q, k_cache, v_cache, o, causal=True, kv_len=lens + 1, q_start=lens, workspace=ws)
        y, h = torch.empty(B, self.C, device=DEV), torch.empty(B, self.C, device=DEV)
        mt.linear_fwd(o.view(B, -1), self._weight("wo"), P["bo"], y)
        mt.dropout_fwd(y, x, 0.0, 0, 0, h)
        return h


def main():
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    ap.add_argument("--dtype", choices=["f32", "bf16"], default="f32")
    for name, default in (("steps", 20), ("batch", 4), ("tokens", 1024), ("width", 1024), ("heads", 16), ("kv-heads", 4),
                          ("head-width", 64)):
        ap.add_argument(f"--{name}", type=int, default=default)
    a = ap.parse_args()
    dtype = torch.float32 if a.dtype == "f32" else torch.bfloat16
    blk = AttentionBlock(a.batch, a.tokens, a.width, a.heads, a.kv_heads, a.head_width, dtype)
    g = torch.Generator(DEV)
    g.manual_seed(1)
    x = torch.randn(a.batch * a.tokens, a.width, generator=g, device=DEV)
    # a target the block can move towards: each token's running mean over its sequence
    rows = x.view(a.batch, a.tokens, -1)
    mean = rows.cumsum(1) / torch.arange(1, a.tokens + 1, device=DEV)[None, :, None]
    target = (rows + mean).view(-1, a.width).contiguous()
    lens = torch.full((a.batch,), a.tokens, dtype=torch.int32, device=DEV)
    blk.step(x, target, lens)
    first = blk.loss.item()
    t0 = time.perf_counter()
    for _ in range(a.steps):
        blk.step(x, target, lens)
    last = blk.loss.item()  # waits
    dt = (time.perf_counter() - t0) / a.steps
    print(f"training: loss {first:.5f} -> {last:.5f} in {a.steps} steps, {dt * 1e3:.3f} ms a step, "
          f"{a.batch * a.tokens / dt:.0f} tokens/s")
    cache = [torch.zeros(a.batch, a.tokens, a.kv_heads, a.head_width, dtype=dtype, device=DEV) for _ in range(2)]
    lens = torch.zeros(a.batch, dtype=torch.int32, device=DEV)
    n = min(64, a.tokens)
    t0 = time.perf_counter()
    for i in range(n):
        blk.decode(rows[:, i].contiguous(), *cache, lens)
        lens += 1
    torch.cuda.synchronize()
    print(f"serving: {n} tokens of {a.batch} sequences, {(time.perf_counter() - t0) / n * 1e6:.0f} us a token")


if __name__ == "__main__":
    main()

"""A small language model trained and served with the library's operators alone.

    h = scale E[tokens];   h += attention(norm(h)) in every layer;   logits = norm(h) E^T
    loss = mean cross-entropy against the next tokens, padding left out

The embedding E is the output projection too: its gradient is the product's plus that of the lookup. ``LanguageModel``
holds the parameters, every buffer and workspace of a training step; ``step`` runs forward, loss, backward, clipping by
the norm over all gradients and Adam, ``decode`` one token of each sequence against the layers' caches. fp32 throughout,
or with bf16 products and attention (fp32 parameters, residual stream, logits and statistics).

    python examples/language_model.py [--dtype bf16] [--steps 20] [--vocab 50001] [--layers 2] [--batch 4] ...
"""
from __future__ import annotations

import argparse
import os
import sys
import time

sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))

import torch

from attention_block import DEV, AttentionBlock, _workspace, mt

NORM_EPS = 1e-5


class LanguageModel:
    def __init__(self, vocab, layers, batch, tokens, width, heads, kv_heads, head_width, dtype=torch.float32, p=0.0, lr=1e-3,
                 max_norm=1.0, seed=0):
        B, T, C, M = batch, tokens, width, batch * tokens
        self.V, self.B, self.T, self.C, self.dtype = vocab, B, T, C, dtype
        self.lr, self.max_norm, self.scale, self.t = lr, max_norm, C ** 0.5, 0
        g = torch.Generator(DEV)
        g.manual_seed(seed)
        f32 = dict(device=DEV, dtype=torch.float32)
        act = dict(device=DEV, dtype=dtype)
        self.blocks = [AttentionBlock(B, T, C, heads, kv_heads, head_width, dtype, p, seed=seed + 1 + i) for i in range(layers)]
        # each layer's norm and the last one
        self.params = {"table": torch.randn(vocab, C, generator=g, **f32) / C ** 0.5}
        for i in range(layers + 1):
            self.params[f"w{i}"], self.params[f"b{i}"] = torch.ones(C, **f32), torch.zeros(C, **f32)
        self.grads = {n: torch.zeros_like(t) for n, t in self.params.items()}
        self.m, self.v = ({n: torch.zeros_like(t) for n, t in self.params.items()} for _ in range(2))
        self.table16 = None if dtype == torch.float32 else torch.empty(vocab, C, **act)
        self.h0, self.dh = torch.empty(M, C, **f32), torch.empty(M, C, **f32)
        self.n = [torch.empty(M, C, **act) for _ in range(layers + 1)]
        for b in self.blocks:
            b.dh = self.dh  # the residual stream's gradient, in place from layer to layer
        self.logits, self.dlogits = torch.empty(M, vocab, **f32), torch.empty(M, vocab, **act)
        self.dn, self.loss, self.norm = torch.empty(M, C, **f32), torch.empty(1, **f32), torch.empty(1, **f32)
        ids = torch.empty(B, T, dtype=torch.int32, device=DEV)
        G = self.grads
        self.ws = _workspace(max(
            mt.embedding_bwd_workspace(ids, self.dh, G["table"]), mt.cross_entropy_workspace(self.logits, ids),
            mt.layer_norm_bwd_workspace(self.h0, self.params["w0"], self.dn, self.dh, G["w0"], G["b0"]),
            mt.linear_bwd_workspace(self.n[0], self._table(), self.dlogits, self.dn, G["table"]),
            mt.clip_grad_norm_workspace(self.all_grads())))
        self.refresh()

    def _table(self):
        return self.params["table"] if self.table16 is None else self.table16

    def all_params(self):
        return [*self.params.values(), *(t for b in self.blocks for t in b.params.values())]

    def all_grads(self):
        return [*self.grads.values(), *(t for b in self.blocks for t in b.grads.values())]

    def refresh(self):
        """The bf16 copies of the table and the projections from the parameters (nothing to do in fp32)."""
        if self.table16 is not None:
            AttentionBlock._cast(self.params["table"], self.table16)
        for b in self.blocks:
            b.refresh()

    # ---------------------------------------------------------------------- training
    def stream(self, i):
        """The residual stream before layer i."""
        return self.blocks[i - 1].h if i else self.h0

    def forward(self, ids, lens):
        """ids [B, T] int32 (-1: padding) -> logits [B T, V]."""
        P = self.params
        mt.embedding_fwd(ids, P["table"], self.h0, scale=self.scale)
        for i, b in enumerate(self.blocks):
            mt.layer_norm_fwd(self.stream(i), P[f"w{i}"], P[f"b{i}"], self.n[i], eps=NORM_EPS)
            b.forward(self.n[i], lens, residual=self.stream(i))
        L = len(self.blocks)
        mt.layer_norm_fwd(self.stream(L), P[f"w{L}"], P[f"b{L}"], self.n[L], eps=NORM_EPS)
        mt.linear_fwd(self.n[L], self._table(), None, self.logits)

    def backward(self, ids, targets, lens):
        """The loss against targets [B, T] (-1: does not count) and the gradients of all parameters."""
        P, G, L = self.params, self.grads, len(self.blocks)
        mt.cross_entropy(self.logits, targets, self.loss, None, self.dlogits, workspace=self.ws)
        mt.linear_bwd(self.n[L], self._table(), self.dlogits, self.dn, G["table"], workspace=self.ws)
        mt.layer_norm_bwd(self.stream(L), P[f"w{L}"], self.dn, self.dh, G[f"w{L}"], G[f"b{L}"], eps=NORM_EPS, workspace=self.ws)
        for i in reversed(range(L)):
            self.blocks[i].backward(self.n[i], lens, through=False)
            dw, db = G[f"w{i}"].zero_(), G[f"b{i}"].zero_()
            mt.layer_norm_bwd(self.stream(i), P[f"w{i}"], self.blocks[i].dx, self.dh, dw, db, eps=NORM_EPS, accumulate=True,
                              workspace=self.ws)  # added to what came past the layer
        mt.embedding_bwd(ids, self.dh, G["table"], scale=self.scale, accumulate=True, workspace=self.ws)

    def step(self, ids, targets, lens):
        """One training step; the loss and the gradients' norm stay on the device (self.loss, self.norm)."""
        self.forward(ids, lens)
        self.backward(ids, targets, lens)
        grads = self.all_grads()
        mt.clip_grad_norm(grads, self.max_norm, self.norm, workspace=self.ws)
        self.t += 1
        for b in self.blocks:
            b.t = self.t
        m, v = ([*s.values(), *(t for b in self.blocks for t in getattr(b, n).values())] for n, s in (("m", self.m), ("v", self.v)))
        mt.adam_step(self.all_params(), grads, m, v, self.lr, 0.9, 0.999, 1e-8, self.t)
        self.refresh()

    # ----------------------------------------------------------------------- serving
    def decode(self, ids, caches, lens):
        """One token of each sequence: ids [B] int32 and each layer's (k, v) caches holding lens [B] tokens; returns
        logits [B, V]. The caller counts lens up."""
        B, P, L = ids.shape[0], self.params, len(self.blocks)
        h = torch.empty(B, self.C, device=DEV)
        n = torch.empty(B, self.C, dtype=self.dtype, device=DEV)
        mt.embedding_fwd(ids, P["table"], h, scale=self.scale)
        for i, b in enumerate(self.blocks):
            mt.layer_norm_fwd(h, P[f"w{i}"], P[f"b{i}"], n, eps=NORM_EPS)
            h = b.decode(n, *caches[i], lens, residual=h)
        mt.layer_norm_fwd(h, P[f"w{L}"], P[f"b{L}"], n, eps=NORM_EPS)
        logits = torch.empty(B, self.V, device=DEV)
        mt.linear_fwd(n, self._table(), None, logits)
        return logits


def main():
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    ap.add_argument("--dtype", choices=["f32", "bf16"], default="f32")
    for name, default in (("steps", 20), ("vocab", 50001), ("layers", 2), ("batch", 4), ("tokens", 1024), ("width", 1024),
                          ("heads", 16), ("kv-heads", 4), ("head-width", 64)):
        ap.add_argument(f"--{name}", type=int, default=default)
    a = ap.parse_args()
    dtype = torch.float32 if a.dtype == "f32" else torch.bfloat16
    model = LanguageModel(a.vocab, a.layers, a.batch, a.tokens, a.width, a.heads, a.kv_heads, a.head_width, dtype)
    g = torch.Generator(DEV)
    g.manual_seed(1)
    # sequences that repeat a pattern of 64 tokens; the last one ends early
    ids = torch.randint(0, a.vocab, (a.batch, 64), generator=g, device=DEV, dtype=torch.int32)
    ids = ids.repeat(1, a.tokens // 64 + 1)[:, :a.tokens + 1].contiguous()
    lens = torch.full((a.batch,), a.tokens, dtype=torch.int32, device=DEV)
    lens[-1] = (a.tokens + 1) // 2
    counts = torch.arange(a.tokens, device=DEV) < lens[:, None]
    tokens, targets = (torch.where(counts, t, -1).int() for t in (ids[:, :-1], ids[:, 1:]))
    model.step(tokens, targets, lens)
    first = model.loss.item()
    t0 = time.perf_counter()
    for _ in range(a.steps):
        model.step(tokens, targets, lens)
    last = model.loss.item()  # waits
    dt = (time.perf_counter() - t0) / a.steps
    print(f"training: loss {first:.4f} -> {last:.4f} in {a.steps} steps, gradient norm {model.norm.item():.3f}, "
          f"{dt * 1e3:.3f} ms a step, {a.batch * a.tokens / dt:.0f} tokens/s")
    caches = [[torch.zeros(a.batch, a.tokens, a.kv_heads, a.head_width, dtype=dtype, device=DEV) for _ in range(2)]
              for _ in model.blocks]
    lens = torch.zeros(a.batch, dtype=torch.int32, device=DEV)
    token, n = ids[:, 0].contiguous(), min(64, a.tokens)
    t0 = time.perf_counter()
    for _ in range(n):
        token = model.decode(token, caches, lens).argmax(-1).int()
        lens += 1
    torch.cuda.synchronize()
    print(f"serving: {n} tokens of {a.batch} sequences, {(time.perf_counter() - t0) / n * 1e6:.0f} us a token")


if __name__ == "__main__":
    main()

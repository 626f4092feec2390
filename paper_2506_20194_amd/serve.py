"""Serve pruned decoder blocks: prompts of different lengths packed one behind the
other, then a token per request, over a paged key-value cache.

One step takes a batch of sequences a number of tokens further, each from the
length that it has in the cache: whole prompts, the next chunks of prompts, or one
token each.  `Step` works out once, for all layers, where the step's tokens stand
and where they go; `run_block` carries their hidden states through one LLaMA-style
block (RMSNorm, rotary attention with grouped heads, SiLU-gated MLP) in the
library's own kernels:

  prompts and chunks   rotate, write K and V into the cache, attend to the packed
                       sequences (duo_attention_packed); K and V come back from the
                       cache where earlier tokens are needed, or where the cache is
                       quantised, so that every token sees what later ones will
  single tokens        rotate, write, attend over the pages (duo_attention_paged)

Weights are a Linear's n x k bf16 matrix or, for single tokens, the compressed
columns of a pruned layer (duo.dsc_compress).  Every linear's input is sparsified
per token with p_x, the calibration rule, when it is given.
"""

from __future__ import annotations

import torch

from . import duo


class Step:
    """The tokens of one step: sequence s goes from before[s] cached tokens to
    before[s] + new[s] (Python ints).  table: int32, row s holds the pages of
    sequence s, enough for its new length.  The token rows of the step are the
    sequences' new tokens one behind the other.  A sequence that needs a page which
    the cache does not have gets NaN for them; the table is read on the device only."""

    def __init__(self, cache, table, before, new):
        if len(before) != len(new) or len(new) != table.shape[0]:
            raise ValueError("Step: before, new and table must name the same sequences")
        if any(b < 0 or n < 0 for b, n in zip(before, new)):
            raise ValueError("Step: lengths must not be negative")
        after = [b + n for b, n in zip(before, new)]
        self.max_len = max(after, default=0)
        if self.max_len > table.shape[1] * cache.page_size:
            raise ValueError("Step: table has too few pages for the new lengths")
        dev = table.device
        self.table, self.m = table, sum(new)
        self.single = all(n == 1 for n in new)
        seq, pos = self._tokens(before, new)
        self.pos = pos.to(dev, torch.int32)
        self.slots = cache.slots(table, seq.to(dev), pos.to(dev))
        if self.single:
            self.lens = torch.tensor(after, dtype=torch.int32).to(dev)
            return
        self.cu_q = self._offsets(new).to(dev)
        # token rows of sequences whose tokens do not all have a page; duo_kv_write skips such
        # tokens and duo_kv_read gives zeros for them, which attention would take for keys
        need = torch.arange(table.shape[1]) * cache.page_size < torch.tensor(after, dtype=torch.int64)[:, None]
        outside = (table < 0) | (table >= cache.data.shape[0])
        self.lost = (outside & need.to(dev)).any(1)[seq.to(dev)][:, None]
        # the whole sequences, where the chunk's own rows of K and V are not all of them
        self.cu_k, self.all_slots = None, self.slots
        if any(before):
            seq, pos = self._tokens([0] * len(after), after)
            self.cu_k, self.all_slots = self._offsets(after).to(dev), cache.slots(table, seq.to(dev), pos.to(dev))

    @staticmethod
    def _tokens(first, count):
        n = torch.tensor(count, dtype=torch.int64)
        seq = torch.repeat_interleave(torch.arange(len(count)), n)
        start = torch.tensor(first, dtype=torch.int64) - (n.cumsum(0) - n)
        return seq, start[seq] + torch.arange(int(n.sum()))

    @staticmethod
    def _offsets(count):
        cu = torch.zeros(len(count) + 1, dtype=torch.int32)
        cu[1:] = torch.tensor(count, dtype=torch.int64).cumsum(0)
        return cu


def linear(x, W, p_x=None, R=None):
    """x W^T (+ R), the rows of x sparsified with p_x first."""
    if isinstance(W, dict):  # compressed columns: a token at a time, sparsified by the GEMV
        y = torch.stack([duo.dsc_gemv(W, row, p_x) for row in x])
        return (y if R is None else y + R.float()).bfloat16()
    if p_x:
        x = duo.duo_act_sparsify(x, p_x)
    return duo.duo_linear(x, W, R=R)


def attention(x, weights, cfg, cache, step, p_x=None):
    """The attention of one block for the step's rows x (already normalised): K and V
    go into the cache, and the heads' outputs are returned."""
    heads, kv, hd, theta = cfg["heads"], cache.kv_heads, cache.head_dim, cfg["theta"]
    q, k, v = (linear(x, weights[nm], p_x) for nm in "qkv")
    duo.duo_rope_at(q, heads, hd, step.pos, theta, out=q)
    duo.duo_rope_at(k, kv, hd, step.pos, theta, out=k)
    duo.duo_kv_write(cache, k, v, step.slots)
    if step.single:
        return duo.duo_attention_paged(q, cache, step.table, step.lens, heads, max_len=step.max_len)
    if step.cu_k is not None or cache.fmt != "bf16":
        k, v = duo.duo_kv_read(cache, step.all_slots)
    a = duo.duo_attention_packed(q, k, v, step.cu_q, heads, kv, hd, cu_k=step.cu_k)
    return a.masked_fill_(step.lost, float("nan"))  # as duo_attention_paged does by itself


def run_block(h, weights, cfg, cache, step, p_x=None):
    """One decoder block for the step's rows: h (step.m x d bf16) -> the same shape.
    weights: q, k, v, o, gate, up, down; cfg: dict(heads, theta, eps); cache: this
    block's (its kv_heads and head_dim are the block's)."""
    if h.shape[0] != step.m:
        raise ValueError("run_block: h must hold the step's tokens")
    if step.m == 0:
        return h.clone()
    a = attention(duo.duo_rmsnorm(h, cfg["eps"]), weights, cfg, cache, step, p_x)
    h2 = linear(a, weights["o"], p_x, R=h)
    x2 = duo.duo_rmsnorm(h2, cfg["eps"])
    m = duo.duo_silu_mul(linear(x2, weights["gate"], p_x), linear(x2, weights["up"], p_x))
    return linear(m, weights["down"], p_x, R=h2)

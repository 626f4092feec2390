"""Serve pruned decoder blocks: prompts of different lengths packed one behind the
other, then a token per request, over a paged key-value cache.

One step takes a batch of sequences a number of tokens further, each from the
length that it has in the cache: whole prompts, the next chunks of prompts, or one
token each.  `Step` works out once, for all layers, where the step's tokens stand
and where they go; `run_block` carries their hidden states through one LLaMA-style
block (RMSNorm, rotary attention with grouped heads, SiLU-gated MLP) in the
library's own kernels:

  every step           rotate queries and keys, with norms of their heads where the block
                       has them, and write K and V into the cache (duo_kv_append)
  whole prompts        attend to the packed sequences (duo_attention_packed)
  chunks, mixed steps  attend over the pages as they are stored (duo_attention_chunk), and
                       so do prompts where the cache is quantised, so that every token
                       sees what later ones will; where the sequences bring many rows or
                       have few tokens (reads_back), K and V come back from the cache
                       (duo_kv_read) and the packed attention takes them in order
  single tokens        attend over the pages (duo_attention_paged)
  a window             duo_attention_chunk for all of them


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
    the cache does not have gets NaN for them (in a block with a window those tokens
    that see one of its tokens: pages that a window has left behind need not be
    there); the table is read on the device only."""

    def __init__(self, cache, table, before, new):
        if len(before) != len(new) or len(new) != table.shape[0]:
            raise ValueError("Step: before, new and table must name the same sequences")
        if any(b < 0 or n < 0 for b, n in zip(before, new)):
            raise ValueError("Step: lengths must not be negative")
        after = [b + n for b, n in zip(before, new)]
        self.max_len, self.max_new = max(after, default=0), max(new, default=0)
        if self.max_len > table.shape[1] * cache.page_size:
            raise ValueError("Step: table has too few pages for the new lengths")
        dev = table.device
        self.table, self.m = table, sum(new)
        self.single = all(n == 1 for n in new)
        seq, pos = self._tokens(before, new)
        self.pos = pos.to(dev, torch.int32)
        self.slots = cache.slots(table, seq.to(dev), pos.to(dev))
        self.lens = torch.tensor(after, dtype=torch.int32).to(dev)
        self.cu_q = torch.arange(self.m + 1, dtype=torch.int32, device=dev) if self.single else self._offsets(new).to(dev)
        self.fewest = min((n for n in new if n), default=0)
        self.cached, self.tokens = any(before), sum(after)
        if self.single:
            return
        # token rows of sequences whose tokens do not all have a page; duo_kv_write skips such
        # tokens and duo_kv_read gives zeros for them, which attention would take for keys
        need = torch.arange(table.shape[1]) * cache.page_size < torch.tensor(after, dtype=torch.int64)[:, None]
        outside = (table < 0) | (table >= cache.data.shape[0])
        self.lost = (outside & need.to(dev)).any(1)[seq.to(dev)][:, None]
        # offsets and slots of the whole sequences, where the chunk's own rows of K and V are not all of
        # them; here and not where they are used, as that may be while a graph is captured, on another stream,
        # or when the table has gone on
        self.cu_k, self.all_slots = None, self.slots
        if self.cached:
            self.cu_k = self._offsets(after).to(dev)
            seq = torch.repeat_interleave(torch.arange(len(after), device=dev), self.lens.long(), output_size=sum(after))
            self.all_slots = cache.slots(table, seq, torch.arange(len(seq), device=dev) - self.cu_k.long()[seq])

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


# Chunks behind cached tokens, and all of a quantised cache, either attend over the pages or have their sequences'
# rows read back for the packed attention.  Reading costs time for every token that is cached, whatever is new, the
# attention over pages more for each row (a new token and head of a group) and to begin with.  So rows are read back
# from MANY_ROWS (MANY_ROWS_16: a cache of 16 bits) of every sequence on, and where little is cached from
# fewer, a part of these, of some sequence on.  Heads of 128, pages and rows read back, in microseconds:
#   8 bits, 65536 tokens of 8 K/V heads, 64 rows 106 and 156, 512 220 and 233, 768 311 and 286, 1024 398 and 351
#   up to 2^18 tokens times K/V heads (32768 of 8): 256 rows 92 and 99, 384 112 and 109, 512 128 and 127, 1024 218 and 185
#   up to 2^17 (16384 of 8): 32 rows 37 and 56 (16 bits), 64 55 and 54, 128 73 and 61, 1024 129 and 106; 4 of 4096: 32 35
#   and 43, 64 49 and 53, 128 66 and 54; 2048: 32 21 and 26 (16 bits), 64 31 and 27, 512 51 and 31; a chunk of 512 on 2048 and
#   three single tokens 105 and 59
#   16 bits, 16384 tokens of 8, 512 rows 71 and 82, 2048 177 and 185, 8192 533 and 523, 16384 1013 and 971
#   up to 1.5 2^16 (4096 of 8): 32 rows 25 and 31, 64 42 and 32, 128 41 and 33, 1024 54 and 52; 16 sequences, chunks of 256 on
#   1024 beside single tokens 74 and 43
# (Rows read back of a quantised cache are rounded to bf16: a root mean square error of the output of 0.003 to
# 0.005, of codes 0.0018.)
MANY_ROWS, MANY_ROWS_16 = 768, 8192


def reads_back(step, cache, heads):
    """Are a chunk's sequences read back for the packed attention?"""
    size, fewest, most = step.tokens * cache.kv_heads, (step.fewest * heads) // cache.kv_heads, (step.max_new * heads) // cache.kv_heads
    if cache.fmt == "bf16":
        return fewest >= MANY_ROWS_16 or size <= 3 << 15 and most >= MANY_ROWS_16 >> 7
    return fewest >= MANY_ROWS or size <= 1 << 18 and most >= MANY_ROWS >> 1 or size <= 1 << 17 and most >= MANY_ROWS >> 4


def attention(x, weights, cfg, cache, step, p_x=None):
    """The attention of one block for the step's rows x (already normalised): K and V
    go into the cache, and the heads' outputs are returned."""
    heads, kv, hd, theta = cfg["heads"], cache.kv_heads, cache.head_dim, cfg["theta"]
    window, sinks = cfg.get("window"), cfg.get("sinks", 0)
    q_gain, k_gain = weights.get("q_norm"), weights.get("k_norm")
    normed = q_gain is not None
    if normed != (k_gain is not None):
        raise ValueError("attention: q_norm and k_norm go together (ones for a norm without gains)")
    q, k, v = (linear(x, weights[nm], p_x) for nm in "qkv")
    duo.duo_kv_append(cache, k, v, step.slots, step.pos, theta, eps=cfg["eps"] if normed else None, k_gain=k_gain, Q=q,
                      q_gain=q_gain, out=q)
    if step.single and not window:
        return duo.duo_attention_paged(q, cache, step.table, step.lens, heads, max_len=step.max_len)
    quantised = cache.fmt != "bf16"
    if window or (step.cached or quantised) and not reads_back(step, cache, heads):
        a = duo.duo_attention_chunk(q, cache, step.table, step.lens, step.cu_q, heads, window=window, sinks=sinks,
                                    max_q=step.max_new, max_len=step.max_len)
        if window:
            return a
    else:
        if quantised or step.cached:
            k, v = duo.duo_kv_read(cache, step.all_slots)
        elif normed:
            duo.duo_head_norm_rope(k, kv, hd, step.pos, k_gain, cfg["eps"], theta, out=k)
        else:
            duo.duo_rope_at(k, kv, hd, step.pos, theta, out=k)
        a = duo.duo_attention_packed(q, k, v, step.cu_q, heads, kv, hd, cu_k=step.cu_k)
    return a.masked_fill_(step.lost, float("nan"))  # as duo_attention_paged does by itself


def run_block(h, weights, cfg, cache, step, p_x=None):
    """One decoder block for the step's rows: h (step.m x d bf16) -> the same shape.
    weights: q, k, v, o, gate, up, down, and q_norm, k_norm where the heads of queries and
    keys are normed before the rotation (head_dim gains each, one dtype, both or neither); cfg:
    dict(heads, theta, eps), and window, sinks where a token sees the last `window`
    ones and the first `sinks` alone; cache: this block's (its kv_heads and head_dim
    are the block's)."""
    if h.shape[0] != step.m:
        raise ValueError("run_block: h must hold the step's tokens")
    if step.m == 0:
        return h.clone()
    a = attention(duo.duo_rmsnorm(h, cfg["eps"]), weights, cfg, cache, step, p_x)
    h2 = linear(a, weights["o"], p_x, R=h)
    x2 = duo.duo_rmsnorm(h2, cfg["eps"])
    m = duo.duo_silu_mul(linear(x2, weights["gate"], p_x), linear(x2, weights["up"], p_x))
    return linear(m, weights["down"], p_x, R=h2)

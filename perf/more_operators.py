"""Operators of a serving step around the paged key-value cache, as cases that can
be timed and compared: norms of query and key heads with the rotation in one pass,
a step's new keys and values rotated on their way into the cache, and attention of
new tokens (chunks of prompts, drafts that are verified, single tokens) over the
pages as they are stored, with a sliding window and first tokens that stay visible
where a model has them.

A case is a dict of plain values; its "op" says which operator one pass goes
through:

  norm    duo.duo_head_norm_rope: every head of every row divided by its root mean
          square, times the gains, and rotated by its token's position
  append  duo.duo_kv_append: keys (with "norm" as above) rotated and written into
          their slots with the values, and the step's queries rotated beside them.  A
          16-bit cache is returned as the numbers it holds; of an 8- or 4-bit one the
          slots just written are read back (duo.duo_kv_read)
  chunk   duo.duo_attention_chunk: the new tokens of a batch of sequences over
          their pages.  Query i of n new ones on a sequence of L tokens (the new ones
          among them) is at position p = L - n + i and sees the tokens up to p; with
          a window of w those after p - w, and the first "sinks" ones

The cache is one byte tensor (pages, K/V heads, block): a block holds page_size
rows of K, as many of V, then for 8 and 4 bits the scales of both, one bfloat16 per
32 channels of a row.  Codes are stored with 128 (a byte) or 8 (half a byte, the
lower half first) added; they are codes of bfloat16 rows, as the keys are that
every other operator on them takes.  Pages that a window has left behind are given
back: their places in a sequence's table hold -1.
"""

from __future__ import annotations

import math
import random

import torch

own = False

DEV = "cuda:0"
THETA = 1e4
EPS = 1e-5
GROUP = 32
BITS = {"bf16": 16, "int8": 8, "int4": 4}


def listed():
    return [
        # The query heads of one decoding step of 64 requests: latency.
        dict(name="norm_step", op="norm", tokens=64, heads=64, hd=128, longest=8192),
        # The same heads over a ragged batch of prompts.
        dict(name="norm_prompts", op="norm", tokens=16411, heads=64, hd=128, longest=2048),
        # One decoding step of 32 requests, 64 query heads on 8: latency.
        dict(name="append_step", op="append", tokens=32, each=1, heads=64, kv=8, hd=128, norm=1, page=16, fmt="bf16",
             pool=16384, longest=8192),
        # Prompts into an 8-bit cache, head norms before the rotation.
        dict(name="append_prompts_int8", op="append", tokens=16411, each=0, heads=64, kv=8, hd=128, norm=1, page=64,
             fmt="int8", pool=20480, longest=2048),
        # A chunk of a long prompt into a 4-bit cache, 32 heads of 64 on 8, no norms.
        dict(name="append_chunk_int4", op="append", tokens=8191, each=0, heads=32, kv=8, hd=64, norm=0, page=64,
             fmt="int4", pool=16384, longest=65536),
        # A short question behind a short conversation, 32 heads on 32: latency.
        dict(name="chunk_short", op="chunk", nseq=1, singles=0, longest=17, context=300, heads=32, kv=32, hd=128, page=16,
             fmt="bf16", window=0, sinks=0, seed=1),
        # Drafts of up to five tokens verified for 32 requests.
        dict(name="chunk_drafts", op="chunk", nseq=32, singles=0, longest=5, context=8192, heads=64, kv=8, hd=128, page=64,
             fmt="bf16", window=0, sinks=0, seed=2),
        # A step that carries two prompts' chunks beside 46 single tokens, 8 bits.
        dict(name="chunk_mixed_int8", op="chunk", nseq=48, singles=46, longest=1024, context=8192, heads=64, kv=8, hd=128,
             page=64, fmt="int8", window=0, sinks=0, seed=3),
        # The next chunk of two long prompts: up to 2048 tokens over up to 16384.
        dict(name="chunk_long", op="chunk", nseq=2, singles=0, longest=2048, context=14336, heads=64, kv=8, hd=128, page=64,
             fmt="bf16", window=0, sinks=0, seed=4),
        # A chunk over a very long context in 4 bits.
        dict(name="chunk_long_int4", op="chunk", nseq=1, singles=0, longest=509, context=65536, heads=32, kv=8, hd=128,
             page=64, fmt="int4", window=0, sinks=0, seed=5),
        # A whole long prompt of a model with a window of 1024 and four sinks.
        dict(name="window_prompt", op="chunk", nseq=1, singles=0, longest=16384, context=0, heads=32, kv=8, hd=128, page=64,
             fmt="bf16", window=1024, sinks=4, seed=6),
        # A decoding step of 64 requests of such a model, 8 bits, contexts of up to 131072.
        dict(name="window_step_int8", op="chunk", nseq=64, singles=64, longest=1, context=131071, heads=64, kv=8, hd=128,
             page=64, fmt="int8", window=4096, sinks=4, seed=7),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


HEADS = ((32, 32), (64, 8), (64, 8), (32, 8), (16, 4), (8, 1), (14, 2), (40, 40), (5, 1), (10, 5), (2, 2))


def draw(rng):
    op = rng.choice(("norm", "append", "append", "chunk", "chunk", "chunk", "chunk", "chunk"))
    heads, kv = rng.choice(HEADS)
    hd = rng.choice((64, 128, 128))
    page = rng.choice((16, 32, 64, 64, 128, 256))
    fmt = rng.choice(("bf16", "int8", "int4"))
    if op == "norm":
        hd = rng.choice((64, 128, 128, 256, 80))
        return dict(op=op, tokens=min(_log(rng, 1, 65536), 2 ** 27 // (heads * hd)), heads=heads, hd=hd,
                    longest=_log(rng, 64, 131072))
    if op == "append":
        tokens = min(_log(rng, 1, 32768), 2 ** 26 // (heads * hd))
        return dict(op=op, tokens=tokens, each=rng.choice((0, 1)), heads=heads, kv=kv, hd=hd, norm=rng.choice((0, 1)),
                    page=page, fmt=fmt, pool=min(16384, 2 ** 25 // (kv * hd)) + 2 * tokens, longest=_log(rng, 64, 131072))
    while True:
        nseq, longest, context = _log(rng, 1, 64), _log(rng, 1, 4096), _log(rng, 1, 65536) - 1
        c = dict(op=op, nseq=nseq, singles=rng.choice((0, 0, nseq, rng.randrange(nseq + 1))), longest=longest,
                 context=context, heads=heads, kv=kv, hd=hd, page=page, fmt=fmt,
                 window=rng.choice((0, 0, 0, _log(rng, 16, 8192))), sinks=rng.choice((0, 4, 4, _log(rng, 1, 200))),
                 seed=rng.randrange(1 << 30))
        if work(c)["flops"] < 9e11 and sum(a + b for a, b in _lengths(c)) * kv * hd < 6e8 \
                and nseq * (context + longest) * kv * hd < 1.5e9:
            return c


# ---------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------

def _lengths(c):
    """(new tokens, tokens before them) of each sequence: the first is the longest,
    the others are spread below it, half of them evenly and half over the logarithm."""
    r = random.Random(c["seed"])

    def spread(lo, hi):
        return r.randint(lo, hi) if r.random() < 0.5 else _log(r, lo, hi)

    out = []
    for i in range(c["nseq"]):
        new = 1 if i >= c["nseq"] - c["singles"] else c["longest"] if i == 0 else spread(1, c["longest"])
        out.append((new, c["context"] if i == 0 else spread(1, c["context"] + 1) - 1))
    return out


def _needed(c, new, before):
    """Tokens [0, a) and [b, end) of a sequence are seen by some new token."""
    end = new + before
    if not c["window"]:
        return 0, 0, end
    b = max(before - c["window"] + 1, 0)
    return min(c["sinks"], b), b, end


def _row_bytes(c):
    return c["hd"] * BITS[c["fmt"]] // 8


def _scale_bytes(c):
    return 0 if c["fmt"] == "bf16" else 2 * c["hd"] // GROUP


def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def _keys(m, c, g):
    """K rows with channels of different sizes (mean square 1), and V rows."""
    s = torch.exp(0.5 * torch.randn(c["kv"] * c["hd"], generator=g, device=DEV))
    s = s / s.square().mean().sqrt()
    K = (torch.randn((m, c["kv"] * c["hd"]), generator=g, device=DEV) * s).bfloat16()
    return K, torch.randn((m, c["kv"] * c["hd"]), generator=g, device=DEV).bfloat16()


def _queries(m, c, g):
    return (torch.randn((m, c["heads"] * c["hd"]), generator=g, device=DEV) * 1.5).bfloat16()


def _gains(c, g):
    return torch.exp(0.3 * torch.randn(c["hd"], generator=g, device=DEV)).bfloat16()


def _cache(pages, c):
    """A pool whose unwritten rows hold what memory may hold: NaN."""
    return torch.full((pages, c["kv"], c["page"] * 2 * (_row_bytes(c) + _scale_bytes(c))), 255, dtype=torch.uint8,
                      device=DEV)


def prepare(case, seed):
    c, g = dict(case), _gen(seed)
    if c["op"] == "norm":
        X = _queries(c["tokens"], c, g)
        pos = torch.randint(0, c["longest"], (c["tokens"],), generator=g, device=DEV, dtype=torch.int32)
        return dict(c=c, X=X, pos=pos, gain=_gains(c, g), Y=torch.empty_like(X))
    if c["op"] == "append":
        m, pages = c["tokens"], -(-c["pool"] // c["page"])
        if c["each"]:  # one token each of that many requests: anywhere in the pool
            slots = torch.randperm(pages * c["page"], generator=g, device=DEV)[:m]
        else:          # whole chunks: pages in any order, filled one after the other
            order = torch.randperm(pages, generator=g, device=DEV)
            t = torch.arange(m, device=DEV)
            slots = order[t // c["page"]] * c["page"] + t % c["page"]
        K, V = _keys(m, c, g)
        Q = _queries(m, c, g)
        pos = torch.randint(0, c["longest"], (m,), generator=g, device=DEV, dtype=torch.int32)
        return dict(c=c, data=_cache(pages, c).zero_(), K=K, V=V, Q=Q, slots=slots.long(), pos=pos, Y=torch.empty_like(Q),
                    k_gain=_gains(c, g) if c["norm"] else None, q_gain=_gains(c, g) if c["norm"] else None)
    lens = _lengths(c)
    p = c["page"]
    # the pages of each sequence that hold a token some query sees
    kept = []
    for new, before in lens:
        a, b, end = _needed(c, new, before)
        n = torch.arange(-(-end // p))
        kept.append(n[(n * p < a) | (n * p + p > b)])
    pages = sum(k.numel() for k in kept) + 8
    order = torch.randperm(pages, generator=g, device=DEV).to(torch.int32)
    table = torch.full((c["nseq"], max(-(-sum(x) // p) for x in lens)), -1, dtype=torch.int32, device=DEV)
    at, slots = 0, []
    for i, k in enumerate(kept):
        mine = order[at:at + k.numel()]
        table[i, k.to(DEV)] = mine
        at += k.numel()
        s = (mine.long()[:, None] * p + torch.arange(p, device=DEV)).view(-1)
        t = (k[:, None] * p + torch.arange(p)).view(-1)
        slots.append(s[(t < sum(lens[i])).to(DEV)])
    slots = torch.cat(slots)
    data = _cache(pages, c)
    for t in range(0, slots.numel(), 65536):
        part = slots[t:t + 65536]
        _store(data, c, *(x.view(-1, c["kv"], c["hd"]) for x in _keys(part.numel(), c, g)), part)
    cu = torch.zeros(c["nseq"] + 1, dtype=torch.int32)
    cu[1:] = torch.tensor([new for new, _ in lens]).cumsum(0)
    Q = _queries(int(cu[-1]), c, g)
    return dict(c=c, Q=Q, data=data, table=table, cu_q=cu.to(DEV), O=torch.empty_like(Q),
                lens=torch.tensor([sum(x) for x in lens], dtype=torch.int32, device=DEV),
                max_q=max(x[0] for x in lens), max_len=max(sum(x) for x in lens))


# ---------------------------------------------------------------------------
# plain forms
# ---------------------------------------------------------------------------

def _parts(data, c):
    """The K rows, V rows, K scales and V scales of a cache, as views."""
    p, rb, sb = c["page"], _row_bytes(c), _scale_bytes(c)
    at = (0, p * rb, 2 * p * rb, 2 * p * rb + p * sb)
    K, V = (data[..., a:a + p * rb].unflatten(-1, (p, rb)) for a in at[:2])
    if not sb:
        return K, V, None, None
    return (K, V) + tuple(data[..., a:a + p * sb].unflatten(-1, (p, sb)) for a in at[2:])


def _coded(X, c):
    """bfloat16 rows (m, kv, hd) as cache bytes and scale bytes."""
    if c["fmt"] == "bf16":
        return X.contiguous().view(torch.uint8), None
    most = 2 ** (BITS[c["fmt"]] - 1) - 1
    x = X.float().unflatten(-1, (-1, GROUP))
    s = (x.abs().amax(-1, keepdim=True) / most).bfloat16()
    s = torch.where(s.float() < 2.0 ** -126, torch.zeros_like(s), s)
    q = torch.where(s > 0, torch.round(x / s.float()), 0.0).clamp(-most, most)
    q = (q + (most + 1)).to(torch.uint8).flatten(-2)
    if c["fmt"] == "int4":
        q = q[..., 0::2] | (q[..., 1::2] << 4)
    return q, s.squeeze(-1).contiguous().view(torch.uint8)


def _store(data, c, K, V, slots):
    page, off = slots // c["page"], slots % c["page"]
    kr, vr, ks, vs = _parts(data, c)
    k, sk = _coded(K, c)
    v, sv = _coded(V, c)
    kr[page, :, off] = k
    vr[page, :, off] = v
    if sk is not None:
        ks[page, :, off] = sk
        vs[page, :, off] = sv


def _numbers(rows, scales, c):
    """Gathered cache bytes (n, kv, row) as float32 numbers (n, kv, hd)."""
    if c["fmt"] == "bf16":
        return rows.view(torch.bfloat16).float()
    if c["fmt"] == "int4":
        rows = torch.stack((rows & 15, rows >> 4), -1).flatten(-2)
    most = 2 ** (BITS[c["fmt"]] - 1)
    x = (rows.float() - most).unflatten(-1, (-1, GROUP))
    return (x * scales.view(torch.bfloat16).float().unsqueeze(-1)).flatten(-2)


def _load(data, c, slots):
    page, off = slots // c["page"], slots % c["page"]
    kr, vr, ks, vs = _parts(data, c)
    if ks is None:
        return _numbers(kr[page, :, off], None, c), _numbers(vr[page, :, off], None, c)
    return _numbers(kr[page, :, off], ks[page, :, off], c), _numbers(vr[page, :, off], vs[page, :, off], c)


def _turned(X, heads, hd, pos, gain, norm):
    """Heads of bfloat16 rows divided by their root mean square (with norm), times
    the gains, rotated: bfloat16 rows (m, heads, hd)."""
    x = X.view(-1, heads, hd).float()
    if norm:
        x = x * torch.rsqrt(x.square().mean(-1, keepdim=True) + EPS) * gain.float()
    f = THETA ** (-2.0 * torch.arange(hd // 2, device=DEV, dtype=torch.float64) / hd)
    a = pos.double()[:, None] * f  # an angle of 1e5 has no place for its fraction in 32 bits
    cos, sin = a.cos().float()[:, None], a.sin().float()[:, None]
    x, y = x.chunk(2, -1)
    return torch.cat((x * cos - y * sin, y * cos + x * sin), -1).bfloat16()


def _alike(lens):
    """Sequences with equally many new tokens, which one batch of products can take."""
    groups = {}
    for i, (new, _) in enumerate(lens):
        groups.setdefault(new, []).append(i)
    return groups.items()


def _attend(s):
    c = s["c"]
    kv, hd, p = c["kv"], c["hd"], c["page"]
    G, lens = c["heads"] // c["kv"], _lengths(c)
    O = torch.empty_like(s["Q"])
    for new, which in _alike(lens):
        n, at = len(which), torch.tensor(which).to(DEV)
        end = s["lens"][at].long()[:, None]
        first = end - new                                     # position of the first new token
        if c["window"]:
            # the sinks, then the window's tokens, padded to the longest of the batch
            b = (first - c["window"] + 1).clamp(min=0)
            a = torch.clamp(b, max=c["sinks"])
            i = torch.arange(min(max(sum(lens[j]) for j in which), c["sinks"] + c["window"] + new - 1), device=DEV)
            t = torch.where(i < a, i, i - a + b)
        else:
            t = torch.arange(max(sum(lens[j]) for j in which), device=DEV).expand(n, -1)
        slots = torch.where(t < end, t, end - 1)              # padding: the last token again, unseen
        slots = torch.gather(s["table"][at].long(), 1, slots // p) * p + slots % p
        k, v = (x.view(n, -1, kv, hd).transpose(1, 2) for x in _load(s["data"], c, slots.view(-1)))
        rows = s["cu_q"][at].long()[:, None] + torch.arange(new, device=DEV)
        q = s["Q"][rows].float().view(n, new, kv, G, hd).permute(0, 2, 3, 1, 4).reshape(n, kv, G * new, hd)
        pos = (first + torch.arange(new, device=DEV))[:, :, None]
        seen = (t[:, None] <= pos) & (t < end)[:, None]
        if c["window"]:
            seen &= (t[:, None] > pos - c["window"]) | (t[:, None] < c["sinks"])
        x = torch.matmul(q, k.transpose(-1, -2).contiguous()).view(n, kv, G, new, -1)
        x = x.mul_(1.0 / math.sqrt(hd)).masked_fill_(~seen[:, None, None], float("-inf"))
        x = x.sub_(x.amax(-1, keepdim=True)).exp_()           # every token sees itself at least
        total = x.sum(-1, keepdim=True)
        o = torch.matmul(x.view(n, kv, G * new, -1), v.contiguous()).view(n, kv, G, new, hd) / total
        O[rows] = o.permute(0, 3, 1, 2, 4).reshape(n, new, -1).bfloat16()
    return O


def _plain(s):
    c = s["c"]
    if c["op"] == "norm":
        return _turned(s["X"], c["heads"], c["hd"], s["pos"], s["gain"], True).flatten(1)
    if c["op"] == "append":
        K = _turned(s["K"], c["kv"], c["hd"], s["pos"], s["k_gain"], c["norm"])
        _store(s["data"], c, K, s["V"].view(K.shape), s["slots"])
        Q = _turned(s["Q"], c["heads"], c["hd"], s["pos"], s["q_gain"], c["norm"]).flatten(1)
        if c["fmt"] == "bf16":
            return Q, s["data"].view(torch.bfloat16)
        return (Q,) + tuple(x.flatten(1).bfloat16() for x in _load(s["data"], c, s["slots"]))
    return _attend(s)


def run(s):
    if not own:
        return _plain(s)
    from paper_2506_20194_amd import duo

    c = s["c"]
    if c["op"] == "norm":
        return duo.duo_head_norm_rope(s["X"], c["heads"], c["hd"], s["pos"], s["gain"], EPS, THETA, out=s["Y"])
    cache = duo.KVCache(s["data"], c["page"], c["kv"], c["hd"], c["fmt"])
    if c["op"] == "append":
        Q = duo.duo_kv_append(cache, s["K"], s["V"], s["slots"], s["pos"], THETA, eps=EPS if c["norm"] else None,
                              k_gain=s["k_gain"], Q=s["Q"], q_gain=s["q_gain"], out=s["Y"])
        return (Q, s["data"].view(torch.bfloat16)) if c["fmt"] == "bf16" else (Q,) + tuple(duo.duo_kv_read(cache, s["slots"]))
    return duo.duo_attention_chunk(s["Q"], cache, s["table"], s["lens"], s["cu_q"], c["heads"],
                                   window=c["window"] or None, sinks=c["sinks"], max_q=s["max_q"], max_len=s["max_len"],
                                   out=s["O"])


# ---------------------------------------------------------------------------
# what a pass cannot do without
# ---------------------------------------------------------------------------

def work(case):
    c = case
    if c["op"] == "norm":
        n = c["tokens"] * c["heads"] * c["hd"]
        return dict(bytes=4.0 * n + 4 * c["tokens"], flops=7.0 * n)
    if c["op"] == "append":
        q, k = c["tokens"] * c["heads"] * c["hd"], c["tokens"] * c["kv"] * c["hd"]
        stored = 2.0 * c["tokens"] * c["kv"] * (_row_bytes(c) + _scale_bytes(c))
        back = 0.0 if c["fmt"] == "bf16" else stored + 4.0 * k  # read back
        return dict(bytes=4.0 * q + 4.0 * k + stored + back + 12 * c["tokens"], flops=(7.0 if c["norm"] else 3.0) * (q + k))
    tokens, keys, pairs = 0, 0, 0
    for new, before in _lengths(c):
        a, b, end = _needed(c, new, before)
        tokens, keys = tokens + new, keys + a + end - b
        if not c["window"]:
            pairs += new * before + new * (new + 1) // 2
            continue
        w = c["window"]
        cut = min(max(w - 1 - before, 0), new)  # queries with fewer than w tokens up to themselves
        pairs += cut * before + cut * (cut + 1) // 2 + (new - cut) * w
        # what the sinks add for the others: min(sinks, tokens before the window)
        x, y = before + cut - w + 1, before + new - w  # of the first and the last of them
        if new > cut:
            low = min(max(c["sinks"] - x, 0), y - x + 1)
            pairs += low * x + low * (low - 1) // 2 + (y - x + 1 - low) * c["sinks"]
    row = 2.0 * c["kv"] * (_row_bytes(c) + _scale_bytes(c))
    return dict(bytes=row * keys + 4.0 * tokens * c["heads"] * c["hd"], flops=4.0 * pairs * c["heads"] * c["hd"])


# ---------------------------------------------------------------------------
# the same in 64 bits
# ---------------------------------------------------------------------------

def _half64(bits):
    """bfloat16 bit patterns as float64."""
    sign = 1.0 - 2.0 * (bits >> 15).double()
    e, f = (bits >> 7) & 255, (bits & 127).double()
    return sign * torch.where(e == 0, f / 128 * 2.0 ** -126, (1 + f / 128) * torch.exp2(e.double() - 127))


def _cached64(data, c, slots, h):
    """K and V numbers of head h at the given slots, from the raw bytes."""
    p, rb, sb = c["page"], _row_bytes(c), _scale_bytes(c)
    base, off = slots // p * data.stride(0) + h * data.stride(1), slots % p
    flat, out = data.view(-1), []
    for which in (0, 1):
        row = base + which * p * rb + off * rb
        b = flat[row[:, None] + torch.arange(rb, device=DEV)].to(torch.int64)
        if c["fmt"] == "bf16":
            out.append(_half64(b[:, 0::2] + 256 * b[:, 1::2]))
            continue
        at = base + 2 * p * rb + which * p * sb + off * sb
        s = flat[at[:, None] + torch.arange(sb, device=DEV)].to(torch.int64)
        s = _half64(s[:, 0::2] + 256 * s[:, 1::2])
        x = torch.empty((slots.numel(), c["hd"]), dtype=torch.float64, device=DEV)
        if c["fmt"] == "int8":
            x.copy_(b - 128)
        else:
            x[:, 0::2], x[:, 1::2] = b % 16 - 8, b // 16 - 8
        for i in range(s.shape[1]):
            x[:, GROUP * i:GROUP * (i + 1)] *= s[:, i:i + 1]
        out.append(x)
    return out


def _rounded64(x):
    """To eight significant bits, ties to even."""
    m, e = torch.frexp(x)
    return torch.round(m * 256) * torch.exp2((e - 8).double())


def _stored64(x, c):
    """What the cache holds for rows of eight significant bits."""
    if c["fmt"] == "bf16":
        return x
    most = {"int8": 127, "int4": 7}[c["fmt"]]
    out = torch.empty_like(x)
    for a in range(0, x.shape[1], GROUP):
        g = x[:, a:a + GROUP]
        s = _rounded64(g.abs().amax(1, keepdim=True) / most)
        out[:, a:a + GROUP] = torch.where(s > 0, torch.round(g / torch.where(s > 0, s, 1.0)), 0.0) * s
    return out


def _turned64(X, heads, hd, pos, gain):
    """The definition channel by channel: rows (m, heads hd) in float64."""
    out = torch.empty(X.shape, dtype=torch.float64, device=DEV)
    half = hd // 2
    for h in range(heads):
        x = X[:, h * hd:(h + 1) * hd].double()
        if gain is not None:
            x = x / torch.sqrt(x.pow(2).sum(1, keepdim=True) / hd + EPS) * gain.double()
        for i in range(half):
            a = pos.double() * THETA ** (-2.0 * i / hd)
            z = torch.complex(x[:, i], x[:, i + half]) * torch.polar(torch.ones_like(a), a)
            out[:, h * hd + i], out[:, h * hd + i + half] = z.real, z.imag
    return out


def exact(case, seed):
    c = case
    s = prepare(case, seed)
    if c["op"] == "norm":
        return _turned64(s["X"], c["heads"], c["hd"], s["pos"], s["gain"])
    if c["op"] == "append":
        Q = _turned64(s["Q"], c["heads"], c["hd"], s["pos"], s["q_gain"])
        K, V = _turned64(s["K"], c["kv"], c["hd"], s["pos"], s["k_gain"]), s["V"].double()
        if c["fmt"] != "bf16":
            return Q, _stored64(_rounded64(K), c), _stored64(V, c)
        out = s["data"].view(torch.bfloat16).double()
        page, off = s["slots"] // c["page"], s["slots"] % c["page"]
        for which, x in enumerate((K, V)):
            for h in range(c["kv"]):
                at = (which * c["page"] + off) * c["hd"]
                out[page[:, None], h, at[:, None] + torch.arange(c["hd"], device=DEV)] = x[:, h * c["hd"]:(h + 1) * c["hd"]]
        return Q, out
    if sum(new * (new + before) for new, before in _lengths(c)) * c["heads"] * c["hd"] > 2e12:  # 64-bit products
        return None
    hd, p, G = c["hd"], c["page"], c["heads"] // c["kv"]
    O = torch.zeros(s["Q"].shape, dtype=torch.float64, device=DEV)
    row = 0
    for r, (new, before) in enumerate(_lengths(c)):
        a, b, end = _needed(c, new, before)
        t = torch.tensor(list(range(a)) + list(range(b, end)), device=DEV)
        slots = s["table"][r].long()[t // p] * p + t % p
        i = before + torch.arange(new, device=DEV)[:, None]
        hidden = t > i
        if c["window"]:
            hidden |= (t <= i - c["window"]) & (t >= c["sinks"])
        for h in range(c["kv"]):
            K, V = _cached64(s["data"], c, slots, h)
            for j in range(h * G, (h + 1) * G):
                q = s["Q"][row:row + new, j * hd:(j + 1) * hd].double()
                x = (q @ K.t() / math.sqrt(hd)).masked_fill_(hidden, float("-inf"))
                O[row:row + new, j * hd:(j + 1) * hd] = torch.softmax(x, 1) @ V
        row += new
    return O

"""The operators that serve a pruned model, as cases that can be timed and
compared: rotation by given positions, a paged key-value cache that is written,
quantised and read back, causal attention over packed prompts with grouped
heads, and attention of one new token per request over the paged cache.

A case is a dict of plain values; its "op" says which operator one pass goes
through:

  rope    duo.duo_rope_at: the rows of X rotated by their tokens' positions
  write   duo.duo_kv_write: K and V rows of new tokens into their slots of the
          cache.  A 16-bit cache is returned as the numbers it holds; an 8- or
          4-bit one is read back at the slots just written (duo.duo_kv_read), as
          a chunk that attends to what its cache holds does
  read    duo.duo_kv_read: cached tokens back as bf16 rows
  packed  duo.duo_attention_packed: causal attention of the prompts (or the next
          chunks of prompts) of a batch, packed one behind the other
  paged   duo.duo_attention_paged: one new token per request over its pages

The cache is one byte tensor (pages, K/V heads, block): a block holds
page_size rows of K, as many of V, then for 8 and 4 bits the scales of both, one
bfloat16 per 32 channels of a row.  Codes are stored with 128 (a byte) or 8 (half
a byte, the lower half first) added.
"""

from __future__ import annotations

import math
import random

import torch

own = False

DEV = "cuda:0"
THETA = 1e4
GROUP = 32
BITS = {"bf16": 16, "int8": 8, "int4": 4}


def listed():
    return [
        # Queries of one decoding step of 64 requests, 64 heads of 128: latency.
        dict(name="rope_step", op="rope", tokens=64, heads=64, hd=128, longest=8192),
        # The same heads over sixteen prompts of 2048.
        dict(name="rope_prompts", op="rope", tokens=32768, heads=64, hd=128, longest=2048),
        # One decoding step of 32 requests: each one's new K and V, eight heads.
        dict(name="write_step", op="write", tokens=32, each=1, kv=8, hd=128, page=16, fmt="bf16", pool=32768),
        # A ragged batch of prompts into an 8-bit cache, and back for its attention.
        dict(name="write_prompts_int8", op="write", tokens=16411, each=0, kv=8, hd=128, page=64, fmt="int8", pool=32768),
        # The cached prefix of one request, 8 bits, 32 heads.
        dict(name="read_prefix_int8", op="read", tokens=2001, kv=32, hd=128, page=16, fmt="int8", pool=8192),
        # A long context out of a 4-bit cache, as its next chunk needs it.
        dict(name="read_long_int4", op="read", tokens=131072, kv=8, hd=128, page=64, fmt="int4", pool=140000),
        # A few short questions, as many K/V heads as query heads: latency.
        dict(name="packed_short", op="packed", nseq=6, longest=96, context=0, heads=32, kv=32, hd=128, seed=1),
        # Prompts of 1 to 2048 tokens, 64 query heads on 8.
        dict(name="packed_ragged", op="packed", nseq=16, longest=2048, context=0, heads=64, kv=8, hd=128, seed=2),
        # The next chunk of two long prompts: 2048 queries over up to 16384 keys.
        dict(name="packed_long_chunks", op="packed", nseq=2, longest=2048, context=14336, heads=64, kv=8, hd=128, seed=3),
        # One request, 1777 tokens so far, 32 heads on 32: latency.
        dict(name="paged_one_request", op="paged", nseq=1, longest=1777, heads=32, kv=32, hd=128, page=16, fmt="bf16", seed=4),
        # A serving batch at very different lengths, 8 bits.
        dict(name="paged_batch_int8", op="paged", nseq=48, longest=8192, heads=64, kv=8, hd=128, page=64, fmt="int8", seed=5),
        # Eight long contexts, the longest of 131072 tokens, 4 bits.
        dict(name="paged_long_int4", op="paged", nseq=8, longest=131072, heads=64, kv=8, hd=128, page=64, fmt="int4", seed=6),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


HEADS = ((32, 32), (64, 8), (64, 8), (32, 8), (16, 4), (8, 1), (12, 4), (40, 40), (5, 1), (10, 5), (2, 2))


def draw(rng):
    op = rng.choice(("rope", "write", "read", "packed", "packed", "packed", "paged", "paged", "paged"))
    heads, kv = rng.choice(HEADS)
    hd = rng.choice((64, 128, 128))
    page = rng.choice((16, 32, 64, 64, 128, 256))
    fmt = rng.choice(("bf16", "int8", "int4"))
    if op == "rope":
        return dict(op=op, tokens=min(_log(rng, 1, 65536), 2 ** 28 // (heads * hd)), heads=heads, hd=hd,
                    longest=_log(rng, 64, 131072))
    if op == "write":
        tokens = _log(rng, 1, 32768)
        return dict(op=op, tokens=tokens, each=rng.choice((0, 1)), kv=kv, hd=hd, page=page, fmt=fmt,
                    pool=min(32768, 2 ** 26 // (kv * hd)) + 2 * tokens)
    if op == "read":
        tokens = min(_log(rng, 1, 131072), 2 ** 27 // (kv * hd))
        return dict(op=op, tokens=tokens, kv=kv, hd=hd, page=page, fmt=fmt, pool=tokens + 4096)
    if op == "packed":
        while True:
            nseq, longest = _log(rng, 1, 64), _log(rng, 1, 4096)
            context = rng.choice((0, 0, _log(rng, 1, 14336)))
            if nseq * heads * longest * (longest + context) < 4.3e9:
                return dict(op=op, nseq=nseq, longest=longest, context=context, heads=heads, kv=kv, hd=hd,
                            seed=rng.randrange(1 << 30))
    while True:
        nseq, longest = _log(rng, 1, 128), _log(rng, 1, 131072)
        if nseq * longest * kv * hd < 1.1e9:
            return dict(op=op, nseq=nseq, longest=longest, heads=heads, kv=kv, hd=hd, page=page, fmt=fmt,
                        seed=rng.randrange(1 << 30))


# ---------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------

def _lengths(c):
    """Tokens of each sequence: the longest, and the others spread over the
    logarithm below it; packed: (new tokens, tokens before them) of each."""
    r = random.Random(c["seed"])
    new = [c["longest"]] + [_log(r, 1, c["longest"]) for _ in range(c["nseq"] - 1)]
    if c["op"] == "paged":
        return new
    before = [c["context"]] + [r.randrange(c["context"] + 1) for _ in range(c["nseq"] - 1)]
    return list(zip(new, before))


def _row_bytes(c):
    return c["hd"] * BITS[c["fmt"]] // 8


def _scale_bytes(c):
    return 0 if c["fmt"] == "bf16" else 2 * c["hd"] // GROUP


def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def _keys(m, c, g):
    """K rows with channels of different sizes, as rotated keys have them (mean
    square 1), and V rows."""
    s = torch.exp(0.5 * torch.randn(c["kv"] * c["hd"], generator=g, device=DEV))
    s = s / s.square().mean().sqrt()
    K = (torch.randn((m, c["kv"] * c["hd"]), generator=g, device=DEV) * s).bfloat16()
    return K, torch.randn((m, c["kv"] * c["hd"]), generator=g, device=DEV).bfloat16()


def _queries(m, c, g):
    return (torch.randn((m, c["heads"] * c["hd"]), generator=g, device=DEV) * 1.5).bfloat16()


def _cache(pages, c):
    """A pool whose unwritten rows hold what memory may hold: NaN."""
    return torch.full((pages, c["kv"], c["page"] * 2 * (_row_bytes(c) + _scale_bytes(c))), 255, dtype=torch.uint8,
                      device=DEV)


def _cu(lengths):
    t = torch.zeros(len(lengths) + 1, dtype=torch.int32)
    t[1:] = torch.tensor(lengths).cumsum(0)
    return t.to(DEV)


def _filled(slots, pages, c, g):
    """A cache that holds rows of K and V at `slots`, written piece by piece."""
    data = _cache(pages, c)
    for t in range(0, slots.numel(), 32768):
        part = slots[t:t + 32768]
        _store(data, c, *_keys(part.numel(), c, g), part)
    return data


def prepare(case, seed):
    c, g = dict(case), _gen(seed)
    if c["op"] == "rope":
        m, d = c["tokens"], c["heads"] * c["hd"]
        X = torch.randn((m, d), generator=g, device=DEV).bfloat16()
        pos = torch.randint(0, c["longest"], (m,), generator=g, device=DEV, dtype=torch.int32)
        return dict(c=c, X=X, pos=pos, Y=torch.empty_like(X))
    if c["op"] == "write":
        pages = -(-c["pool"] // c["page"])
        if c["each"]:  # one token each of that many requests: anywhere in the pool
            slots = torch.randperm(pages * c["page"], generator=g, device=DEV)[:c["tokens"]]
        else:          # whole prompts: pages in any order, filled one after the other
            order = torch.randperm(pages, generator=g, device=DEV)
            t = torch.arange(c["tokens"], device=DEV)
            slots = order[t // c["page"]] * c["page"] + t % c["page"]
        K, V = _keys(c["tokens"], c, g)
        data = _cache(pages, c).zero_()
        return dict(c=c, data=data, K=K, V=V, slots=slots.long())
    if c["op"] == "read":
        pages = -(-c["pool"] // c["page"])
        order = torch.randperm(pages, generator=g, device=DEV)
        t = torch.arange(c["tokens"], device=DEV)
        slots = order[t // c["page"]] * c["page"] + t % c["page"]
        return dict(c=c, data=_filled(slots, pages, c, g), slots=slots)
    if c["op"] == "packed":
        new, before = zip(*_lengths(c))
        every = [a + b for a, b in zip(new, before)]
        Q = _queries(sum(new), c, g)
        K, V = _keys(sum(every), c, g)
        return dict(c=c, Q=Q, K=K, V=V, cu_q=_cu(new), cu_k=_cu(every) if c["context"] else None,
                    longest=max(every), O=torch.empty_like(Q))
    lens = _lengths(c)
    need = [-(-n // c["page"]) for n in lens]
    pages = sum(need) + 8
    order = torch.randperm(pages, generator=g, device=DEV).to(torch.int32)
    table = torch.zeros((c["nseq"], max(need)), dtype=torch.int32, device=DEV)
    at = 0
    for i, n in enumerate(need):
        table[i, :n] = order[at:at + n]
        at += n
    t = torch.cat([torch.arange(n, device=DEV) + i * max(need) * c["page"] for i, n in enumerate(lens)])
    slots = table.view(-1)[t // c["page"]].long() * c["page"] + t % c["page"]
    data = _filled(slots, pages, c, g)
    return dict(c=c, Q=_queries(c["nseq"], c, g), data=data, table=table,
                lens=torch.tensor(lens, dtype=torch.int32, device=DEV))


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
    """Rows (m, kv, hd) in float32 as cache bytes and scale bytes."""
    if c["fmt"] == "bf16":
        return X.bfloat16().view(torch.uint8), None
    most = 2 ** (BITS[c["fmt"]] - 1) - 1
    x = X.unflatten(-1, (-1, GROUP))
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
    shape = (-1, c["kv"], c["hd"])
    k, sk = _coded(K.view(shape).float(), c)
    v, sv = _coded(V.view(shape).float(), c)
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


def _attend(q, k, v, seen):
    """softmax(q k^T / sqrt(hd)) v over the keys that are seen; 0 where none is."""
    x = torch.matmul(q, k.transpose(-1, -2)) * (1.0 / math.sqrt(q.shape[-1]))
    x = x.masked_fill(~seen, float("-inf"))
    top = x.amax(-1, keepdim=True)
    p = torch.exp(x - torch.where(top == float("-inf"), 0.0, top))
    total = p.sum(-1, keepdim=True)
    return torch.matmul(p, v) / torch.where(total == 0, 1.0, total)


def _plain(s):
    c = s["c"]
    if c["op"] == "rope":
        m, h, hd = c["tokens"], c["heads"], c["hd"]
        f = THETA ** (-2.0 * torch.arange(hd // 2, device=DEV, dtype=torch.float64) / hd)
        a = s["pos"].double()[:, None] * f  # an angle of 1e5 has no place for its fraction in 32 bits
        cos, sin = a.cos().float()[:, None], a.sin().float()[:, None]
        x, y = s["X"].view(m, h, 2, hd // 2).float().unbind(2)
        return torch.stack((x * cos - y * sin, y * cos + x * sin), 2).view(m, h * hd).bfloat16()
    if c["op"] == "write":
        _store(s["data"], c, s["K"], s["V"], s["slots"])
        if c["fmt"] == "bf16":
            return s["data"].view(torch.bfloat16)
        return tuple(x.flatten(1).bfloat16() for x in _load(s["data"], c, s["slots"]))
    if c["op"] == "read":
        return tuple(x.flatten(1).bfloat16() for x in _load(s["data"], c, s["slots"]))
    kv, hd, n = c["kv"], c["hd"], c["nseq"]
    G = c["heads"] // kv
    if c["op"] == "paged":
        L = c["longest"]
        t = torch.arange(L, device=DEV)
        live = t < s["lens"][:, None]
        slots = s["table"].long()[:, t // c["page"]] * c["page"] + t % c["page"]
        k, v = _load(s["data"], c, torch.where(live, slots, slots[:, :1]).view(-1))
        k, v = (x.view(n, L, kv, hd).transpose(1, 2) for x in (k, v))
        q = s["Q"].float().view(n, kv, G, hd)
        return _attend(q, k, v, live[:, None, None]).reshape(n, c["heads"] * hd).bfloat16()
    # packed: sequences side by side, padded to the longest
    cu_q = s["cu_q"].long()
    cu_k = cu_q if s["cu_k"] is None else s["cu_k"].long()
    lq, lk = cu_q.diff()[:, None], cu_k.diff()[:, None]
    i, j = torch.arange(c["longest"], device=DEV), torch.arange(s["longest"], device=DEV)
    rows = cu_q[:-1, None] + torch.minimum(i, lq - 1)
    cols = cu_k[:-1, None] + torch.minimum(j, lk - 1)
    q = s["Q"].float()[rows].view(n, -1, kv, G, hd).permute(0, 2, 3, 1, 4).reshape(n, kv, -1, hd)
    k, v = (x.float()[cols].view(n, -1, kv, hd).transpose(1, 2) for x in (s["K"], s["V"]))
    seen = (j <= (i + lk - lq)[:, :, None]) & (j < lk)[:, None]
    o = _attend(q, k, v, seen[:, None].repeat(1, 1, G, 1))
    o = o.view(n, kv, G, -1, hd).permute(0, 3, 1, 2, 4).reshape(n, c["longest"], c["heads"] * hd)
    return o[i < lq].bfloat16()


def run(s):
    if not own:
        return _plain(s)
    from paper_2506_20194_amd import duo

    c = s["c"]
    if c["op"] == "rope":
        return duo.duo_rope_at(s["X"], c["heads"], c["hd"], s["pos"], THETA, out=s["Y"])
    if c["op"] == "packed":
        return duo.duo_attention_packed(s["Q"], s["K"], s["V"], s["cu_q"], c["heads"], c["kv"], c["hd"],
                                        cu_k=s["cu_k"], out=s["O"])
    cache = duo.KVCache(s["data"], c["page"], c["kv"], c["hd"], c["fmt"])
    if c["op"] == "write":
        duo.duo_kv_write(cache, s["K"], s["V"], s["slots"])
        return s["data"].view(torch.bfloat16) if c["fmt"] == "bf16" else duo.duo_kv_read(cache, s["slots"])
    if c["op"] == "read":
        return duo.duo_kv_read(cache, s["slots"])
    return duo.duo_attention_paged(s["Q"], cache, s["table"], s["lens"], c["heads"], max_len=c["longest"])


# ---------------------------------------------------------------------------
# what a pass cannot do without
# ---------------------------------------------------------------------------

def work(case):
    c = case
    if c["op"] == "rope":
        n = c["tokens"] * c["heads"] * c["hd"]
        return dict(bytes=4.0 * n + 4 * c["tokens"], flops=3.0 * n)
    if c["op"] in ("write", "read"):
        n = c["tokens"] * c["kv"]
        rows, stored = 4.0 * n * c["hd"], 2.0 * n * (_row_bytes(c) + _scale_bytes(c))
        both = 2 if c["op"] == "write" and c["fmt"] != "bf16" else 1  # written, then read back
        return dict(bytes=both * (rows + stored) + 8 * c["tokens"], flops=2.0 * both * n * c["hd"])
    if c["op"] == "paged":
        n = sum(_lengths(c))
        return dict(bytes=2.0 * n * c["kv"] * (_row_bytes(c) + _scale_bytes(c)) + 4.0 * c["nseq"] * c["heads"] * c["hd"],
                    flops=4.0 * n * c["heads"] * c["hd"])
    tokens, keys, pairs = 0, 0, 0
    for new, before in _lengths(c):
        tokens, keys = tokens + new, keys + new + before
        pairs += new * before + new * (new + 1) // 2
    return dict(bytes=4.0 * (tokens * c["heads"] + keys * c["kv"]) * c["hd"], flops=4.0 * pairs * c["heads"] * c["hd"])


# ---------------------------------------------------------------------------
# the same in 64 bits
# ---------------------------------------------------------------------------

def _cached64(data, c, slots):
    """K and V numbers of the given slots, head by head from the raw bytes."""
    hd, p, rb, sb = c["hd"], c["page"], _row_bytes(c), _scale_bytes(c)
    base = slots // p * data.stride(0)
    off = slots % p
    out = []
    flat = data.view(-1)
    for which in (0, 1):
        x = torch.empty((slots.numel(), c["kv"], hd), dtype=torch.float64, device=DEV)
        for h in range(c["kv"]):
            row = base + h * data.stride(1) + which * p * rb + off * rb
            b = flat[row[:, None] + torch.arange(rb, device=DEV)].to(torch.int64)
            if c["fmt"] == "bf16":
                x[:, h] = _half64(b[:, 0::2] + 256 * b[:, 1::2])
                continue
            at = base + h * data.stride(1) + 2 * p * rb + which * p * sb + off * sb
            s = flat[at[:, None] + torch.arange(sb, device=DEV)].to(torch.int64)
            s = _half64(s[:, 0::2] + 256 * s[:, 1::2]).repeat_interleave(GROUP, 1)
            if c["fmt"] == "int8":
                x[:, h] = (b - 128) * s
            else:
                x[:, h, 0::2] = (b % 16 - 8) * s[:, 0::2]
                x[:, h, 1::2] = (b // 16 - 8) * s[:, 1::2]
        out.append(x)
    return out


def _half64(bits):
    """bfloat16 bit patterns as float64."""
    sign = 1.0 - 2.0 * (bits >> 15).double()
    e, f = (bits >> 7) & 255, (bits & 127).double()
    return sign * torch.where(e == 0, f / 128 * 2.0 ** -126, (1 + f / 128) * torch.exp2(e.double() - 127))


def _stored64(X, c):
    """What the cache holds for rows X (m, kv hd)."""
    x = X.double()
    if c["fmt"] == "bf16":
        return x
    most = {"int8": 127, "int4": 7}[c["fmt"]]
    for a in range(0, x.shape[1], GROUP):
        g = x[:, a:a + GROUP]
        m, e = torch.frexp(g.abs().amax(1, keepdim=True) / most)
        s = torch.ldexp(torch.round(m * 256), e - 8)  # eight significant bits
        g.copy_(torch.where(s > 0, torch.round(g / torch.where(s > 0, s, 1.0)), 0.0) * s)
    return x


def exact(case, seed):
    c = case
    s = prepare(case, seed)
    if c["op"] == "rope":
        m, half = c["tokens"], c["hd"] // 2
        out = torch.empty((m, c["heads"] * c["hd"]), dtype=torch.float64, device=DEV)
        for i in range(half):
            a = s["pos"].double() * THETA ** (-2.0 * i / c["hd"])
            z = torch.polar(torch.ones_like(a), a)[:, None]
            z = z * torch.complex(s["X"][:, i::c["hd"]].double(), s["X"][:, i + half::c["hd"]].double())
            out[:, i::c["hd"]], out[:, i + half::c["hd"]] = z.real, z.imag
        return out
    if c["op"] == "write":
        K, V = _stored64(s["K"], c), _stored64(s["V"], c)
        if c["fmt"] != "bf16":
            return K, V
        out = s["data"].view(torch.bfloat16).double()
        page, off = s["slots"] // c["page"], s["slots"] % c["page"]
        for which, x in enumerate((K, V)):
            for h in range(c["kv"]):
                at = (which * c["page"] + off) * c["hd"]
                out[page[:, None], h, at[:, None] + torch.arange(c["hd"], device=DEV)] = x[:, h * c["hd"]:(h + 1) * c["hd"]]
        return out
    if c["op"] == "read":
        return tuple(x.flatten(1) for x in _cached64(s["data"], c, s["slots"]))
    hd, G = c["hd"], c["heads"] // c["kv"]
    O = torch.zeros(s["Q"].shape, dtype=torch.float64, device=DEV)
    if c["op"] == "paged":
        for r, n in enumerate(_lengths(c)):
            t = torch.arange(n, device=DEV)
            K, V = _cached64(s["data"], c, s["table"][r].long()[t // c["page"]] * c["page"] + t % c["page"])
            for h in range(c["heads"]):
                q = s["Q"][r, h * hd:(h + 1) * hd].double()
                O[r, h * hd:(h + 1) * hd] = torch.softmax((K[:, h // G] @ q) / math.sqrt(hd), 0) @ V[:, h // G]
        return O
    a = b = 0
    for new, before in _lengths(c):
        n = new + before
        later = torch.ones((new, n), dtype=torch.bool, device=DEV).triu_(before + 1)
        for h in range(c["heads"]):
            K, V = (s[x][b:b + n, h // G * hd:(h // G + 1) * hd].double() for x in "KV")
            q = s["Q"][a:a + new, h * hd:(h + 1) * hd].double()
            O[a:a + new, h * hd:(h + 1) * hd] = (q @ K.t() / math.sqrt(hd)).masked_fill_(later, float("-inf")).softmax(-1) @ V
        a, b = a + new, b + n
    return O

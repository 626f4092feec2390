"""Attention of new tokens over the paged cache on the GPU, against the float64 reference
on the numbers that the cache stands for, with the bound that the reference derives
(oracle/serve_ref.py).  In 8 and 4 bits codes are multiplied exactly, with an offset, whose error
is that of the paged attention's tests, or as fp16 numbers, which codes of 8 bits are rounded
to: 2^-11 of each product in a score (a code's product with its scale has up to 15 bits, fp16
eleven, and half of its last one is 2^-11 of a number just above a power of two), and of each value,
which the bound of a probability's rounding to bf16 covers (2^-8; fp16's two roundings are 2^-10)."""

import numpy as np
import pytest
import torch

from oracle import serve_ref as S

pytestmark = pytest.mark.gpu
DEV = torch.device("cuda:0")
FMTS = ["bf16", "int8", "int4"]


def say(*a):
    print("[case]", *a, flush=True)


def f64(t):
    return t.detach().cpu().double().numpy()


def bf(shape, seed, scale=1.0):
    return (torch.randn(shape, generator=torch.Generator().manual_seed(seed)) * scale).bfloat16()


def seen(lq, n, window, sinks):
    p, j = np.arange(lq)[:, None] + n - lq, np.arange(n)[None, :]
    s = j <= p
    return s if not window else s & ((j > p - window) | (j < sinks))


class Batch:
    """Sequences of (new tokens, all tokens) in scattered pages of a cache whose other bytes are
    255 (NaN), pages that no query sees neither in the cache nor in the table."""

    def __init__(self, d, seqs, heads, kv, hd, page, fmt, window=0, sinks=0, seed=0, q_scale=1.5, touch=None):
        self.d, self.seqs, self.window, self.sinks = d, seqs, window, sinks
        self.heads, self.kv, self.hd, self.fmt = heads, kv, hd, fmt
        g = torch.Generator().manual_seed(seed + 100)
        lens = [n for _, n in seqs]
        need = [-(-n // page) for n in lens]
        order = torch.randperm(sum(need) + 3, generator=g)
        table = torch.full((len(seqs), max(max(need), 1)), -1, dtype=torch.int32)
        at, slots = 0, []
        for i, (lq, n) in enumerate(seqs):
            some = seen(lq, n, window, sinks).any(0)
            for t in range(need[i]):
                if lq == 0 or some[t * page:t * page + page].any():
                    table[i, t] = order[at]
                    at += 1
            t = torch.arange(n)
            slots.append(torch.where(table[i, t // page] < 0, -1, table[i, t // page].long() * page + t % page))
        self.slots = torch.cat(slots) if slots else torch.zeros(0, dtype=torch.int64)
        self.cache = d.KVCache.empty(len(order), page, kv, hd, fmt, DEV)
        self.cache.data.fill_(255)
        T = sum(lens)
        self.K, self.V = bf((T, kv * hd), seed + 1), bf((T, kv * hd), seed + 2)
        if touch:
            touch(self)
        if T:
            d.duo_kv_write(self.cache, self.K.to(DEV), self.V.to(DEV), self.slots.long().to(DEV))
        self.table = table.to(DEV)
        self.lens = torch.tensor(lens, dtype=torch.int32, device=DEV)
        cu = torch.zeros(len(seqs) + 1, dtype=torch.int32)
        cu[1:] = torch.tensor([lq for lq, _ in seqs]).cumsum(0)
        self.cu = cu.to(DEV)
        self.Q = bf((int(cu[-1]), heads * hd), seed + 3, q_scale)

    def run(self, scale=None, pad=0, **kw):
        w = self.heads * self.hd
        Qd = torch.empty((len(self.Q), w + pad), dtype=torch.bfloat16, device=DEV)[:, :w]
        Qd.copy_(self.Q)
        out = torch.full((len(self.Q) + 2, w + (3 if pad else 0)), 9.0, dtype=torch.bfloat16, device=DEV)
        O = out[:len(self.Q), :w]
        kw.setdefault("max_q", max((lq for lq, _ in self.seqs), default=0))
        self.d.duo_attention_chunk(Qd, self.cache, self.table, self.lens, self.cu, self.heads, window=self.window or None,
                                   sinks=self.sinks, scale=scale, out=O, **kw)
        assert (out[:, w:] == 9.0).all() and (out[len(self.Q):] == 9.0).all()
        return O

    def check(self, O, scale=None, skip=()):
        heads, kv, hd = self.heads, self.kv, self.hd
        scale = hd ** -0.5 if scale is None else scale
        at = row = 0
        worst = 0.0
        for i, (lq, n) in enumerate(self.seqs):
            k, v = (f64(t)[at:at + n].reshape(n, kv, hd) for t in (self.K, self.V))
            q = f64(self.Q)[row:row + lq].reshape(lq, heads, hd)
            o = f64(O)[row:row + lq].reshape(lq, heads, hd)
            at, row = at + n, row + lq
            if lq == 0 or i in skip:
                continue
            see = seen(lq, n, self.window, self.sinks)
            k, v = (np.where(see.any(0)[:, None, None], t, 0.0) for t in (k, v))
            err = lambda ref: float((np.abs(o - ref[0]) / ref[1]).max(initial=0.0))
            assert np.isfinite(o).all(), (i, lq, n)
            if self.fmt == "bf16" or n == 0:
                w = err(S.attend(q, k, v, scale, see))
            else:
                (ck, sk), (cv, sv) = S.quantize(k, self.fmt), S.quantize(v, self.fmt)
                k, v = S.numbers(ck, sk), S.numbers(cv, sv)
                G = heads // kv
                qs = np.abs(q).reshape(lq, heads, -1, 32).sum(-1)  # (lq, heads, groups)
                extra = np.einsum("lhg,nhg->lhn", qs, np.repeat(sk, G, 1)) * abs(scale) * 300 * 2.0 ** -24
                X = np.where(see[:, None], np.einsum("lhd,nhd->lhn", q, np.repeat(k, G, 1)) * scale, -np.inf)
                some = see.any(1)[:, None, None]
                p = np.exp(X - np.where(some, X.max(2, keepdims=True, initial=-np.inf), 0.0))
                p = p / np.where(some, p.sum(2, keepdims=True), 1.0)
                add = 2.0 ** -15 * np.repeat(np.einsum("lhn,nhg->lhg", p, np.repeat(sv, G, 1)), 32, -1)
                if self.fmt == "int8":
                    extra = extra + 2.0 ** -11 * np.einsum("lhd,nhd->lhn", np.abs(q), np.repeat(np.abs(k), G, 1)) * abs(scale)
                # Scores off by at most e change p = exp(x) / sum exp(x) by a factor within exp(2 e), of which
                # the reference's bound has the first term, 2 e: where e is not small the rest is added.
                e = np.where(see[:, None], extra, 0.0).max(2)[..., None]
                rest = (np.expm1(2 * e) - 2 * e) * np.einsum("lhn,nhd->lhd", p, np.repeat(np.abs(v), G, 1))
                ref, tol = S.attend(q, k, v, scale, see, extra)
                w = err((ref, tol + add + rest))
            worst = max(worst, w)
        say(f"worst error / bound {worst:.3f}")
        assert worst <= 1


def one(d, seqs, heads, kv, hd, page, fmt, window=0, sinks=0, scale=None, pad=0, seed=0, q_scale=1.5, **kw):
    b = Batch(d, seqs, heads, kv, hd, page, fmt, window, sinks, seed, q_scale)
    O = b.run(scale, pad, **kw)
    b.check(O, scale)
    return b, O


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("heads,kv", [(1, 1), (4, 4), (8, 1), (16, 1), (24, 1), (64, 8), (10, 5), (40, 2), (6, 2), (5, 1), (200, 1)])
def test_heads(duo_lib, heads, kv, hd, fmt):
    say("chunk heads", heads, kv, hd, fmt)
    one(duo_lib, [(3, 70), (1, 1), (17, 130), (1, 90)], heads, kv, hd, 16, fmt)


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("page", [16, 32, 64, 128, 256])
@pytest.mark.parametrize("seqs", [
    [(1, 1)], [(0, 0), (2, 2), (0, 5), (1, 0), (3, 2)], [(15, 16), (16, 16), (1, 17), (31, 31), (32, 33)],
    [(63, 64), (64, 64), (65, 65), (1, 127), (128, 128), (2, 129)], [(255, 257), (33, 511), (1, 513)], [(500, 1000), (3, 3)],
    [(2, 2049), (130, 2048)],
])
def test_lengths(duo_lib, seqs, page, fmt):
    """From no token to a few blocks and tiles; more new tokens than cached ones give zeros first."""
    say("chunk lengths", seqs, page, fmt)
    b, O = one(duo_lib, seqs, 4, 2, 128, page, fmt)
    row = 0
    for lq, n in seqs:
        assert (O[row:row + max(lq - n, 0)] == 0).all()
        row += lq


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 1), (7, 3), (64, 0), (64, 4), (100, 65), (257, 130), (1000, 4), (100000, 4), (33, 5000)])
def test_windows(duo_lib, window, sinks, fmt):
    say("chunk windows", window, sinks, fmt)
    seqs = [(1, 2000), (300, 700), (5, 64), (40, 40), (1, 1), (129, 1500), (2, 3)]
    one(duo_lib, seqs, 4, 2, 64, 16, fmt, window, sinks)
    one(duo_lib, seqs, 8, 1, 128, 64, fmt, window, sinks)


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("hd", [64, 128])
def test_long(duo_lib, hd, fmt):
    say("chunk long", hd, fmt)
    one(duo_lib, [(3, 20011)], 8, 1, hd, 64, fmt)
    one(duo_lib, [(1, 5000), (60, 9000), (0, 0), (7, 16384), (1, 300)], 4, 2, hd, 16, fmt)
    one(duo_lib, [(1, 30000), (70, 20000)], 8, 2, hd, 16, fmt, 5000, 4)


@pytest.mark.parametrize("fmt", FMTS)
def test_many(duo_lib, fmt):
    say("chunk many", fmt)
    one(duo_lib, [(1 + 5 * i % 7, 7 + (37 * i) % 700) for i in range(200)], 8, 2, 128, 32, fmt)
    one(duo_lib, [(1, (37 * i) % 700) for i in range(200)], 8, 2, 128, 32, fmt, 50, 4)
    one(duo_lib, [(2, 2 + i % 90) for i in range(1500)], 4, 4, 64, 16, fmt)
    one(duo_lib, [(1 + 13 * i % 40, 45 + 7 * i % 200) for i in range(150)], 8, 1, 64, 16, fmt)
    one(duo_lib, [(1 + 13 * i % 40, 45 + 7 * i % 200) for i in range(150)], 8, 1, 64, 16, fmt, 30, 4)


@pytest.mark.parametrize("fmt", FMTS)
def test_many_rows(duo_lib, fmt):
    """Chunks of many rows, beside single tokens and short ones, split and whole."""
    say("chunk many rows", fmt)
    one(duo_lib, [(400, 1500), (1, 3000), (77, 77), (1, 5), (300, 301)], 16, 2, 128, 64, fmt)
    one(duo_lib, [(260, 2600), (1, 3000), (9, 400)], 5, 1, 64, 16, fmt)
    one(duo_lib, [(700, 1200), (33, 2000)], 12, 1, 128, 16, fmt, 300, 10)
    one(duo_lib, [(150, 150)], 40, 40, 64, 16, fmt)


@pytest.mark.parametrize("window,sinks", [(0, 0), (150, 70)])
@pytest.mark.parametrize("fmt", FMTS)
def test_very_many_rows(duo_lib, fmt, window, sinks):
    """Sequences of more blocks than there are workgroups (64 heads of 64 on 8), and of more than a thousand
    rows, beside others."""
    say("chunk very many rows", fmt, window, sinks)
    one(duo_lib, [(1, 700), (1100, 1300), (300, 340), (40, 100)], 64, 8, 64, 16, fmt, window, sinks)
    one(duo_lib, [(257, 1000), (70, 600), (512, 512)], 8, 2, 128, 64, fmt, window, sinks)


@pytest.mark.parametrize("fmt", ["int8", "int4"])
@pytest.mark.parametrize("lq", [150, 170])
def test_overlapping_sequences_of_many_rows(duo_lib, fmt, lq):
    """More sequences of many rows than the offsets should allow: rows of one and the same sequence."""
    say("chunk overlapping sequences", fmt)
    d, heads, kv, hd = duo_lib, 16, 2, 64
    b = Batch(d, [(lq, 400)], heads, kv, hd, 16, fmt)
    want = b.run()
    b.check(want)
    cu = torch.tensor([0, lq, 0, lq, 0, lq], dtype=torch.int32, device=DEV)
    table, lens = b.table.repeat(5, 1), b.lens.repeat(5)
    O = d.duo_attention_chunk(b.Q.to(DEV), b.cache, table, lens, cu, heads)
    b.check(O)


@pytest.mark.parametrize("fmt", FMTS)
def test_scale_strides_hints(duo_lib, fmt):
    say("chunk scale, strides, hints", fmt)
    seqs = [(2, 300), (40, 140), (1, 9)]
    one(duo_lib, seqs, 4, 2, 64, 16, fmt, scale=0.4, pad=8)
    one(duo_lib, seqs, 4, 2, 64, 16, fmt, scale=-0.1, max_len=301)
    one(duo_lib, seqs, 4, 2, 128, 16, fmt, scale=0.0, max_len=300)
    one(duo_lib, seqs, 16, 2, 128, 64, fmt, q_scale=60.0)
    for hint in (None, 0, 1, 1000):  # a wrong bound costs time only
        one(duo_lib, seqs, 16, 2, 128, 64, fmt, max_q=hint)


@pytest.mark.parametrize("kind", ["keys", "queries", "values", "small values", "large values", "everything"])
@pytest.mark.parametrize("heads,lq", [(2, 60), (16, 60), (16, 150), (16, 170)])
@pytest.mark.parametrize("fmt", FMTS)
def test_magnitudes(duo_lib, fmt, heads, lq, kind):
    """Keys, values and queries whose sizes differ by many powers of two, and all values
    far from 1."""
    say("chunk magnitudes", fmt, heads, lq, kind)
    g = torch.Generator().manual_seed(5)

    def spread(x, lo, hi, some):
        e = torch.randint(lo, hi + 1, (len(x), 1), generator=g).float()
        x.copy_((x.float() * torch.exp2(torch.where(torch.rand((len(x), 1), generator=g) < some, e, 0.0))).bfloat16())

    def touch(b):
        if kind in ("keys", "everything"):
            spread(b.K, -30, 5, 0.1)
        if kind in ("values", "everything"):
            spread(b.V, -30, 30, 0.1)
        if kind == "small values":
            b.V.mul_(2.0 ** -90)
            b.V[:40] = 0.0
        if kind == "large values":
            b.V.mul_(2.0 ** 70)

    b = Batch(duo_lib, [(lq, 700), (9, 90), (70, 70)], heads, 2, 128, 16, fmt, touch=touch)
    if kind in ("queries", "everything"):
        spread(b.Q, -30, 6, 0.3)
    b.check(b.run())


@pytest.mark.parametrize("top", [0.3, 4.0])
@pytest.mark.parametrize("lq", [2, 60, 170])
@pytest.mark.parametrize("fmt", FMTS)
def test_long_tail(duo_lib, fmt, lq, top):
    """A first token that has nearly all of the probability, 2^21 times any other one's, but zeros in half of
    its channels: there the many others are the output.  Their values lie on either side of its."""
    say("chunk long tail", fmt, lq, top)

    def touch(b):
        b.K.mul_(0.05)
        b.K[0] = 1.28
        g = torch.Generator().manual_seed(9)
        b.V.copy_(torch.rand(b.V.shape, generator=g) * 0.25 - 0.05)
        b.V[0] = 0.0
        b.V[0, ::2] = top

    b = Batch(duo_lib, [(lq, 4000)], 16, 2, 128, 16, fmt, touch=touch)
    b.Q.copy_(1.0 + 0.05 * b.Q)
    b.check(b.run())


@pytest.mark.parametrize("fmt", FMTS)
def test_lengths_and_offsets_are_cut(duo_lib, fmt):
    """Negative lengths are empty, ones past max_len end there; offsets outside Q are cut, rows
    of no sequence are left alone."""
    say("chunk cut lengths", fmt)
    d, heads, kv, hd = duo_lib, 4, 2, 64
    b = Batch(d, [(3, 200), (3, 200), (2, 55)], heads, kv, hd, 16, fmt)
    lens = torch.tensor([-3, 90000, 55], dtype=torch.int32, device=DEV)
    out = torch.full((8, heads * hd), 9.0, dtype=torch.bfloat16, device=DEV)
    d.duo_attention_chunk(b.Q.to(DEV), b.cache, b.table, lens, b.cu, heads, max_len=150, out=out)
    ref = Batch(d, [(3, 0), (3, 150), (2, 55)], heads, kv, hd, 16, fmt)
    rows = torch.cat([torch.arange(200, 350), torch.arange(400, 455)])
    ref.K, ref.V = b.K[rows], b.V[rows]
    ref.check(out)
    assert (out[:3] == 0).all()
    out.fill_(9.0)
    cu = torch.tensor([-5, 2, 2, 100], dtype=torch.int32, device=DEV)  # rows 0, 1 and 2 .. 7
    d.duo_attention_chunk(b.Q.to(DEV), b.cache, b.table, b.lens, cu, heads, out=out)
    ref = Batch(d, [(2, 200), (0, 200), (6, 55)], heads, kv, hd, 16, fmt)
    ref.K, ref.V, ref.Q = b.K, b.V, b.Q
    ref.check(out)
    out.fill_(9.0)
    cu = torch.tensor([1, 3, 2, 5], dtype=torch.int32, device=DEV)  # rows 1, 2; none (falls); 2, 3, 4
    d.duo_attention_chunk(b.Q.to(DEV), b.cache, b.table, b.lens, cu, heads, out=out)
    assert (out[[0, 5, 6, 7]] == 9.0).all() and torch.isfinite(out).all()


@pytest.mark.parametrize("window,sinks", [(0, 0), (40, 4)])
@pytest.mark.parametrize("heads,lq", [(2, 5), (16, 60), (16, 150), (16, 170)])
@pytest.mark.parametrize("fmt", FMTS)
def test_page_outside(duo_lib, fmt, heads, lq, window, sinks):
    """Queries that see a token in a page that is not there are NaN, and only they."""
    say("chunk page outside", fmt, heads, lq, window, sinks)
    seqs = [(lq, 300), (lq, 300), (1, 300), (lq, 300)]
    b = Batch(duo_lib, seqs, heads, 2, 128, 16, fmt, window, sinks)
    good = b.run()
    b.check(good)
    lost = [(0, 18), (2, 17), (3, 0)]
    for i, (s, page) in enumerate(lost):
        b.table[s, page] = (-1, b.cache.data.shape[0], 2 ** 31 - 1)[i]
    O = b.run()
    row = 0
    for s, (n, total) in enumerate(seqs):
        hit = np.zeros(n, dtype=bool)
        for t, page in lost:
            if t == s:
                hit = seen(n, total, window, sinks)[:, 16 * page:16 * page + 16].any(1)
        nan = torch.isnan(O[row:row + n]).all(1).cpu().numpy()
        assert (nan == hit).all(), (s, nan, hit)
        assert torch.equal(O[row:row + n].cpu()[torch.from_numpy(~hit)], good[row:row + n].cpu()[torch.from_numpy(~hit)])
        row += n


@pytest.mark.parametrize("window,sinks", [(0, 0), (20, 3)])
@pytest.mark.parametrize("heads,lq", [(2, 9), (16, 70), (16, 140), (32, 140)])
@pytest.mark.parametrize("fmt", FMTS)
def test_unseen_numbers(duo_lib, fmt, heads, lq, window, sinks):
    """Infinities and NaN in keys and values that a query does not see have no influence on
    it, whoever else sees them; those who see a NaN value are NaN in its channels."""
    say("chunk unseen numbers", fmt, heads, lq, window, sinks)
    n, kv, hd = 150, 2, 64
    clean = Batch(duo_lib, [(lq, n)], heads, kv, hd, 16, fmt, window, sinks)
    good = f64(clean.run())
    j = n - lq // 2  # this token's value is NaN (in 8 and 4 bits its group), and the last token's key

    def touch(b):
        b.V[j, 3] = float("nan")
        b.V[n - 2, hd + 40] = float("inf")
        b.K[n - 1, 5] = float("nan")

    b = Batch(duo_lib, [(lq, n)], heads, kv, hd, 16, fmt, window, sinks, touch=touch)
    O = f64(b.run())
    see = seen(lq, n, window, sinks)
    G = heads // kv
    for h in range(heads):
        o, r = (x.reshape(lq, heads, hd)[:, h] for x in (O, good))
        for i in range(lq):
            bad = np.zeros(hd, dtype=bool)
            if h // G == 0 and see[i, j]:
                bad[3 if fmt == "bf16" else slice(0, 32)] = True
            if h // G == 1 and see[i, n - 2]:
                if fmt == "bf16":
                    assert o[i, 40] == np.inf or np.isnan(o[i, 40])
                bad[40 if fmt == "bf16" else slice(32, 64)] = True
            if h // G == 0 and see[i, n - 1]:
                bad[:] = True
            assert (np.isnan(o[i]) | ~bad | (o[i] == np.inf)).all(), (h, i)
            assert np.isfinite(o[i][~bad]).all() and (np.abs(o[i] - r[i])[~bad] <= 2.0 ** -6).all(), (h, i)


@pytest.mark.parametrize("lq", [90, 170])
def test_repeats_streams_and_graphs(duo_lib, lq):
    """The same bits from any workspace, on another stream and in replayed graphs whose lengths
    change between the replays; two graphs share a workspace."""
    say("chunk repeats, streams, graphs")
    d = duo_lib
    seqs = [(1, 3000), (lq, 700), (4, 500)]
    b = Batch(d, seqs, 16, 2, 128, 64, "int8")
    Q, w = b.Q.to(DEV), 16 * 128
    size = d.attention_chunk_workspace("int8", len(Q), 3, 16, 2, 128, b.table.shape[1] * 64, DEV).numel()
    call = lambda **kw: d.duo_attention_chunk(Q, b.cache, b.table, b.lens, b.cu, 16, **kw)
    first = call(ws=torch.zeros(size, dtype=torch.uint8, device=DEV))
    assert torch.equal(first, call(ws=torch.full((size,), 255, dtype=torch.uint8, device=DEV)))
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        other = call()
    torch.cuda.current_stream().wait_stream(s)
    assert torch.equal(first, other)
    ws = torch.empty(size, dtype=torch.uint8, device=DEV)
    outs, graphs = [torch.empty_like(Q) for _ in range(2)], []
    for o in outs:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            call(ws=ws, out=o)
        graphs.append(g)
    for step in range(3):
        b.lens.sub_(step)
        want = call()
        for o, g in zip(outs, graphs):
            o.fill_(7.0)
            g.replay()
            torch.cuda.synchronize()
            assert torch.equal(o, want)


def test_agrees_with_paged_attention(duo_lib):
    """One new token each: what duo_attention_paged gives, up to the last bit of a sum's order."""
    say("chunk against paged")
    d = duo_lib
    for fmt in FMTS:
        b = Batch(d, [(1, 1 + 97 * i) for i in range(30)], 8, 2, 128, 16, fmt)
        O = b.run()
        P = d.duo_attention_paged(b.Q.to(DEV), b.cache, b.table, b.lens, 8)
        assert ((O.double() - P.double()).abs() <= 2.0 ** -6 * P.double().abs().max()).all()
        b.check(O)


def test_no_rows(duo_lib):
    say("chunk of nothing")
    d = duo_lib
    cache = d.KVCache.empty(2, 16, 1, 64, "bf16", DEV)
    e = lambda *s, t=torch.int32: torch.zeros(s, dtype=t, device=DEV)
    assert d.duo_attention_chunk(e(0, 64, t=torch.bfloat16), cache, e(1, 2), e(1), e(2), 1).shape == (0, 64)
    assert d.duo_attention_chunk(e(0, 64, t=torch.bfloat16), cache, e(0, 2), e(0), e(1), 1).shape == (0, 64)
    for n in (3, 300):  # no pages at all
        O = d.duo_attention_chunk(e(n, 64, t=torch.bfloat16), cache, e(1, 0), e(1), torch.tensor([0, n], device=DEV).int(), 1)
        assert (O == 0).all()

"""Attention of single queries over the paged cache on the GPU, against the float64
reference on the numbers that the cache stands for, with the bound that the
reference derives (oracle/serve_ref.py).  Codes may be multiplied with an offset
of up to 136 (a number of eight bits plus the bias) that is taken out again in
fp32: 300 2^-24 of the scale per query entry and key in a score, and 2^-15 of the
sum of probabilities times scales in the output."""

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


def filled(duo, lens, kv, hd, page, fmt, seed=0, fill=255, k_scale=1.0):
    """A cache that holds sequences of `lens` tokens in scattered pages, every other
    byte of it `fill` (255: NaN), with the table and the K and V that were written."""
    need = [-(-n // page) for n in lens]
    pages = sum(need) + 3
    g = torch.Generator().manual_seed(seed + 100)
    order = torch.randperm(pages, generator=g)
    table = torch.full((len(lens), max(max(need), 1)), -12345, dtype=torch.int32)
    at = 0
    for i, n in enumerate(need):
        table[i, :n] = order[at:at + n].int()
        at += n
    cache = duo.KVCache.empty(pages, page, kv, hd, fmt, DEV)
    cache.data.fill_(fill)
    T = sum(lens)
    K, V = bf((T, kv * hd), seed + 1, k_scale), bf((T, kv * hd), seed + 2)
    if T:
        seq = torch.repeat_interleave(torch.arange(len(lens)), torch.tensor(lens))
        pos = torch.cat([torch.arange(n) for n in lens])
        duo.duo_kv_write(cache, K.to(DEV), V.to(DEV), cache.slots(table, seq, pos).to(DEV))
    return cache, table.to(DEV), K, V


def check(O, Q, K, V, lens, heads, kv, hd, fmt, scale=None):
    scale = hd ** -0.5 if scale is None else scale
    at, worst = 0, 0.0
    for i, n in enumerate(lens):
        k, v = (f64(t)[at:at + n].reshape(n, kv, hd) for t in (K, V))
        at += n
        q = f64(Q)[i].reshape(1, heads, hd)
        extra, add = 0.0, 0.0
        if fmt != "bf16" and n:
            (ck, sk), (cv, sv) = S.quantize(k, fmt), S.quantize(v, fmt)
            k, v = S.numbers(ck, sk), S.numbers(cv, sv)
            G = heads // kv
            qs = np.abs(q[0]).reshape(heads, -1, 32).sum(-1)  # (heads, groups)
            extra = np.einsum("hg,nhg->hn", qs, np.repeat(sk, G, 1))[None] * abs(scale) * 300 * 2.0 ** -24
            S1 = np.einsum("hd,nhd->hn", q[0], np.repeat(k, G, 1)) * scale
            p = np.exp(S1 - S1.max(1, keepdims=True))
            p /= p.sum(1, keepdims=True)
            add = 2.0 ** -15 * np.repeat(np.einsum("hn,nhg->hg", p, np.repeat(sv, G, 1)), 32, -1)
        ref, tol = S.attend(q, k, v, scale, np.ones((1, n), dtype=bool), extra)
        err = np.abs(f64(O)[i].reshape(heads, hd) - ref[0])
        assert np.isfinite(err).all(), (i, n)
        worst = max(worst, float((err / (tol[0] + add)).max(initial=0.0)) if n else float(err.max()) * 1e30)
    say(f"worst error / bound {worst:.3f}")
    assert worst <= 1


def run(duo, lens, heads, kv, hd, page, fmt, scale=None, q_scale=1.5, max_len=None, seed=0, pad=0, k_scale=1.0):
    cache, table, K, V = filled(duo, lens, kv, hd, page, fmt, seed, k_scale=k_scale)
    Q = bf((len(lens), heads * hd), seed + 3, q_scale)
    Qd = torch.empty((len(lens), heads * hd + pad), dtype=torch.bfloat16, device=DEV)[:, :heads * hd]
    Qd.copy_(Q)
    out = torch.full((len(lens), heads * hd + (3 if pad else 0)), 9.0, dtype=torch.bfloat16, device=DEV)
    duo.duo_attention_paged(Qd, cache, table, torch.tensor(lens, dtype=torch.int32, device=DEV), heads, max_len=max_len,
                            scale=scale, out=out[:, :heads * hd])
    assert (out[:, heads * hd:] == 9.0).all()
    check(out[:, :heads * hd], Q, K, V, lens, heads, kv, hd, fmt, scale)


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("heads,kv", [(1, 1), (4, 4), (8, 1), (16, 1), (24, 1), (64, 8), (10, 5), (40, 2), (6, 2)])
def test_heads(duo_lib, heads, kv, hd, fmt):
    say("paged heads", heads, kv, hd, fmt)
    run(duo_lib, [70, 1, 130], heads, kv, hd, 16, fmt)


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("page", [16, 32, 64, 128, 256])
@pytest.mark.parametrize("lens", [[1], [0, 2, 0], [15, 16, 17, 31, 32, 33], [63, 64, 65, 127, 128, 129], [255, 256, 257, 511, 513],
                                  [1000, 3], [2048, 2049]])
def test_lengths(duo_lib, lens, page, fmt):
    say("paged lengths", lens, page, fmt)
    run(duo_lib, lens, 4, 2, 128, page, fmt)


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("hd", [64, 128])
def test_long(duo_lib, hd, fmt):
    say("paged long", hd, fmt)
    run(duo_lib, [20011], 8, 1, hd, 64, fmt)
    run(duo_lib, [5000, 1, 0, 16384, 300], 4, 2, hd, 16, fmt)


@pytest.mark.parametrize("fmt", FMTS)
def test_many(duo_lib, fmt):
    say("paged many", fmt)
    run(duo_lib, [(37 * i) % 700 for i in range(200)], 8, 2, 128, 32, fmt)


@pytest.mark.parametrize("fmt", FMTS)
def test_scale_strides_bound_of_lengths(duo_lib, fmt):
    say("paged scale, strides, max_len", fmt)
    run(duo_lib, [300, 40], 4, 2, 64, 16, fmt, scale=0.4, pad=8)
    run(duo_lib, [300, 40], 4, 2, 64, 16, fmt, scale=-0.1, max_len=301)
    run(duo_lib, [300, 40], 4, 2, 128, 16, fmt, scale=0.0, max_len=300)
    run(duo_lib, [900, 400], 4, 2, 128, 64, fmt, q_scale=60.0)
    run(duo_lib, [900, 400], 4, 2, 128, 64, fmt, k_scale=1e-20)
    run(duo_lib, [0, 0], 4, 2, 128, 64, fmt)


@pytest.mark.parametrize("fmt", FMTS)
def test_lengths_are_cut(duo_lib, fmt):
    """Negative lengths are empty, ones past max_len end there."""
    say("paged cut lengths", fmt)
    cache, table, K, V = filled(duo_lib, [200, 200, 200], 2, 64, 16, fmt)
    Q = bf((3, 256), 3)
    lens = torch.tensor([-3, 90000, 55], dtype=torch.int32, device=DEV)
    O = duo_lib.duo_attention_paged(Q.to(DEV), cache, table, lens, 4, max_len=150)
    rows = torch.cat([torch.arange(200, 350), torch.arange(400, 455)])
    check(O, Q, K[rows], V[rows], [0, 150, 55], 4, 2, 64, fmt)


@pytest.mark.parametrize("fmt", FMTS)
def test_page_outside(duo_lib, fmt):
    """A sequence with a token in a page that is not there is NaN; the others are
    not touched, and entries behind a sequence's end are not read."""
    say("paged page outside", fmt)
    lens = [100, 100, 2000, 40, 100]
    cache, table, K, V = filled(duo_lib, lens, 2, 128, 16, fmt)
    table[0, 6], table[2, 50], table[4, 0] = -1, cache.data.shape[0], 2 ** 31 - 1
    table[1, 7:], table[3, 3:] = 2 ** 31 - 1, -2 ** 31
    Q = bf((5, 4 * 128), 3)
    O = duo_lib.duo_attention_paged(Q.to(DEV), cache, table, torch.tensor(lens, dtype=torch.int32, device=DEV), 4)
    assert torch.isnan(O[[0, 2, 4]]).all()
    check(O[[1, 3]], Q[[1, 3]], torch.cat((K[100:200], K[2200:2240])), torch.cat((V[100:200], V[2200:2240])), [100, 40], 4, 2,
          128, fmt)


@pytest.mark.parametrize("fmt", FMTS)
def test_poisoned_numbers(duo_lib, fmt):
    """A NaN among a sequence's keys makes it NaN, one among its values the channels
    that hold it (in 8 and 4 bits: their group); after its end nothing does."""
    say("paged poisoned", fmt)
    lens, heads, kv, hd = [100, 130], 2, 1, 128
    cache, table, K, V = filled(duo_lib, lens, kv, hd, 16, fmt)
    k, v = K.clone(), V.clone()
    k[10, 3] = float("nan")
    v[100 + 77, 40] = float("nan")
    seq = torch.repeat_interleave(torch.arange(2), torch.tensor(lens))
    pos = torch.cat([torch.arange(n) for n in lens])
    duo_lib.duo_kv_write(cache, k.to(DEV), v.to(DEV), cache.slots(table.cpu(), seq, pos).to(DEV))
    Q = bf((2, heads * hd), 3)
    O = duo_lib.duo_attention_paged(Q.to(DEV), cache, table, torch.tensor(lens, dtype=torch.int32, device=DEV), heads)
    assert torch.isnan(O[0]).all()
    nan = torch.isnan(O[1].view(heads, hd))
    hit = torch.zeros(hd, dtype=torch.bool, device=DEV)
    hit[slice(40, 41) if fmt == "bf16" else slice(32, 64)] = True
    assert (nan == hit).all()
    cut = torch.tensor([10, 77], dtype=torch.int32, device=DEV)
    O = duo_lib.duo_attention_paged(Q.to(DEV), cache, table, cut, heads)
    rows = torch.cat([torch.arange(10), torch.arange(100, 177)])
    check(O, Q, K[rows], V[rows], [10, 77], heads, kv, hd, fmt)


@pytest.mark.parametrize("fmt", FMTS)
def test_offsets_past_32_bits(duo_lib, fmt):
    say("paged offsets past 32 bits", fmt)
    page, kv, hd, heads = 256, 8, 128, 16
    pages = -(-(9 << 29) // duo_lib.kv_page_bytes(page, kv, hd, fmt))
    cache = duo_lib.KVCache.empty(pages, page, kv, hd, fmt, DEV)
    table = torch.tensor([[pages - 1, 0, pages - 2], [1, pages // 2, 2]], dtype=torch.int32)
    lens = [700, 300]
    K, V = bf((1000, kv * hd), 1), bf((1000, kv * hd), 2)
    seq = torch.repeat_interleave(torch.arange(2), torch.tensor(lens))
    pos = torch.cat([torch.arange(n) for n in lens])
    duo_lib.duo_kv_write(cache, K.to(DEV), V.to(DEV), cache.slots(table, seq, pos).to(DEV))
    Q = bf((2, heads * hd), 3)
    O = duo_lib.duo_attention_paged(Q.to(DEV), cache, table.to(DEV), torch.tensor(lens, dtype=torch.int32, device=DEV), heads)
    check(O, Q, K, V, lens, heads, kv, hd, fmt)


def test_infinite_scores(duo_lib):
    """-inf scores weigh nothing; nothing but -inf, or +inf, is NaN."""
    say("paged infinite scores")
    hd, lens = 64, [1, 100, 100]
    cache, table, K, V = filled(duo_lib, lens, 1, hd, 16, "bf16")
    k = K.clone()
    k[0, 0], k[5, 0], k[101 + 50, 0] = float("-inf"), float("-inf"), float("inf")
    seq = torch.repeat_interleave(torch.arange(3), torch.tensor(lens))
    pos = torch.cat([torch.arange(n) for n in lens])
    duo_lib.duo_kv_write(cache, k.to(DEV), V.to(DEV), cache.slots(table.cpu(), seq, pos).to(DEV))
    Q = bf((3, hd), 3)
    Q[:, 0] = 1.0
    O = duo_lib.duo_attention_paged(Q.to(DEV), cache, table, torch.tensor(lens, dtype=torch.int32, device=DEV), 1)
    assert torch.isnan(O[0]).all() and torch.isnan(O[2]).all()
    rows = [i for i in range(1, 101) if i != 5]
    check(O[1:2], Q[1:2], K[rows], V[rows], [99], 1, 1, hd, "bf16")


@pytest.mark.parametrize("fmt", FMTS)
def test_repeats_streams_and_graph(duo_lib, fmt):
    """The same bits again, from a stream of its own, from a workspace that holds
    anything, and from a replayed graph whose lengths and pages change."""
    say("paged repeats, streams, graph", fmt)
    lens, heads, kv, hd = [3000, 50, 0, 777], 16, 2, 128
    cache, table, K, V = filled(duo_lib, lens, kv, hd, 16, fmt)
    Q = bf((4, heads * hd), 3).to(DEV)
    n = torch.tensor(lens, dtype=torch.int32, device=DEV)
    a = duo_lib.duo_attention_paged(Q, cache, table, n, heads)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        b = duo_lib.duo_attention_paged(Q, cache, table, n, heads)
    s.synchronize()
    assert torch.equal(a, b)
    ws = duo_lib.attention_paged_workspace(4, heads, kv, hd, table.shape[1] * 16, DEV)
    ws.fill_(255)
    assert torch.equal(a, duo_lib.duo_attention_paged(Q, cache, table, n, heads, ws=ws))
    out = torch.empty_like(a)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        duo_lib.duo_attention_paged(Q, cache, table, n, heads, out=out, ws=ws)
    for cut in ([3000, 50, 0, 777], [1, 0, 0, 700], [2999, 49, 0, 3], [3000, 50, 0, 777]):
        n.copy_(torch.tensor(cut, dtype=torch.int32))
        want = duo_lib.duo_attention_paged(Q, cache, table, n, heads)
        out.zero_()
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(want, out)
    assert torch.equal(a, out)


def test_refusals(duo_lib):
    say("paged refusals")
    cache, table, K, V = filled(duo_lib, [40, 40], 2, 64, 16, "int8")
    Q = bf((2, 256), 3).to(DEV)
    n = torch.tensor([40, 40], dtype=torch.int32, device=DEV)
    ok = lambda **k: duo_lib.duo_attention_paged(**{**dict(Q=Q, cache=cache, table=table, lens=n, heads=4), **k})
    ok()
    with pytest.raises(TypeError):
        ok(Q=Q.float())
    with pytest.raises(TypeError):
        ok(table=table.long())
    with pytest.raises(TypeError):
        ok(lens=n.long())
    with pytest.raises(ValueError):
        ok(lens=n[:1])
    with pytest.raises(ValueError):
        ok(table=table[:1])
    with pytest.raises(ValueError):
        ok(max_len=table.shape[1] * 16 + 1)
    with pytest.raises(ValueError):
        ok(heads=2)
    with pytest.raises(duo_lib.DuoError):
        ok(heads=3, Q=Q[:, :192])            # no multiple of the cache's heads
    with pytest.raises(duo_lib.DuoError):
        ok(scale=float("inf"))
    with pytest.raises(ValueError):
        ok(Q=Q.cpu())
    with pytest.raises(ValueError):
        duo_lib.KVCache(cache.data[:, :, 1:], 16, 2, 64, "int8")
    with pytest.raises(ValueError):
        duo_lib.KVCache(cache.data, 16, 2, 64, "int3")
    with pytest.raises(duo_lib.DuoError):
        duo_lib.KVCache.empty(4, 24, 2, 64, "int8")
    with pytest.raises(TypeError):
        duo_lib.duo_kv_write(cache, Q[:, :128].contiguous(), Q[:, :128].contiguous(), n)


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("nseq,heads,kv,hd", [(120, 16, 16, 128), (330, 5, 5, 64), (210, 96, 8, 128), (200, 64, 8, 64)])
def test_many_short_rows(duo_lib, nseq, heads, kv, hd, fmt):
    """Rows (sequences times K/V heads) in the thousands, where short ones are done by
    single waves, with longer and empty ones between them."""
    say("paged many short rows", nseq, heads, kv, hd, fmt)
    lens = [(1, 0, 63, 64, 65, 128, 129, 200, 256, 257, 31, 17)[i % 12] for i in range(nseq)]
    lens[7], lens[-1] = 700, 5
    run(duo_lib, lens, heads, kv, hd, 32, fmt, pad=8)

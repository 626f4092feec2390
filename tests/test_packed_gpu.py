"""Attention over packed sequences with grouped heads on the GPU, against the float64
reference with the bound that it derives (oracle/serve_ref.py)."""

import numpy as np
import pytest
import torch

from oracle import serve_ref as S

pytestmark = pytest.mark.gpu
DEV = torch.device("cuda:0")


def say(*a):
    print("[case]", *a, flush=True)


def f64(t):
    return t.detach().cpu().double().numpy()


def bf(shape, seed, scale=1.0):
    return (torch.randn(shape, generator=torch.Generator().manual_seed(seed)) * scale).bfloat16()


def cu(lens, first=0):
    return torch.tensor(np.concatenate(([first], first + np.cumsum(lens))), dtype=torch.int32)


def check(O, Q, K, V, lq, lk, heads, kv, hd, scale=None, q0=0, k0=0):
    """Every sequence of packed float64 arrays against the reference."""
    a, b, worst = q0, k0, 0.0
    for n, m in zip(lq, lk):
        ref, tol = S.attend(Q[a:a + n].reshape(n, heads, hd), K[b:b + m].reshape(m, kv, hd), V[b:b + m].reshape(m, kv, hd),
                            hd ** -0.5 if scale is None else scale, S.causal(n, m))
        err = np.abs(O[a:a + n].reshape(n, heads, hd) - ref)
        assert np.isfinite(err).all(), (n, m)
        worst = max(worst, float((err / tol).max(initial=0.0)))
        a, b = a + n, b + m
    say(f"worst error / bound {worst:.3f}")
    assert worst <= 1


def run(duo, lq, lk, heads, kv, hd, scale=None, q_scale=1.5, pad=0):
    same = lk is None
    lk = lq if same else lk
    Q, K, V = bf((sum(lq), heads * hd), 1, q_scale), bf((sum(lk), kv * hd), 2), bf((sum(lk), kv * hd), 3)
    dev = [torch.empty((t.shape[0], t.shape[1] + pad * (i + 1)), dtype=torch.bfloat16, device=DEV)[:, :t.shape[1]]
           for i, t in enumerate((Q, K, V))]
    for d, t in zip(dev, (Q, K, V)):
        d.copy_(t)
    full = torch.full((sum(lq), heads * hd + (3 if pad else 0)), 9.0, dtype=torch.bfloat16, device=DEV)
    out = full[:, :heads * hd]
    duo.duo_attention_packed(*dev, cu(lq).to(DEV), heads, kv, hd, cu_k=None if same else cu(lk).to(DEV), scale=scale,
                             out=out)
    assert (full[:, heads * hd:] == 9.0).all()
    check(f64(out), f64(Q), f64(K), f64(V), lq, lk, heads, kv, hd, scale)


@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("heads,kv", [(1, 1), (8, 8), (8, 1), (6, 2), (10, 5), (16, 4)])
def test_heads(duo_lib, heads, kv, hd):
    say("packed heads", heads, kv, hd)
    run(duo_lib, [70, 1, 130, 33], None, heads, kv, hd)


@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("lq", [[1], [2], [31, 32, 33], [63, 64, 65], [127, 128, 129], [255, 1, 257], [0, 5, 0, 0, 300, 0],
                                [1] * 150, [513, 7]])
def test_lengths(duo_lib, lq, hd):
    say("packed lengths", lq[:8], hd)
    run(duo_lib, lq, None, 4, 2, hd)


@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("lq,lk", [([1], [1000]), ([1, 1, 1], [64, 65, 1]), ([40, 129], [300, 700]), ([64], [127]),
                                   ([128, 5], [129, 5]), ([3, 130], [513, 4])])
def test_continued(duo_lib, lq, lk, hd):
    """Queries that are the last of longer sequences, and (130 on 4 keys) queries
    before the first key."""
    say("packed continued", lq, lk, hd)
    run(duo_lib, lq, lk, 4, 2, hd)


@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("lq,lk", [([5, 200, 70], [0, 3, 69]), ([64, 1], [0, 0]), ([300], [100])])
def test_rows_without_keys(duo_lib, lq, lk, hd):
    say("rows without keys", lq, lk, hd)
    run(duo_lib, lq, lk, 3, 1, hd)


@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("heads,kv,lq,lk", [(4, 2, [1], [5000]), (8, 8, [3, 40], [4097, 600]), (16, 2, [9, 1, 0, 70], [900, 8200, 3, 130]),
                                            (1, 1, [64], [2048]), (2, 1, [130], [1100]), (4, 4, [5, 300], [2, 3000])])
def test_split_over_keys(duo_lib, heads, kv, lq, lk, hd):
    say("split over keys", heads, kv, lq, lk, hd)
    assert duo_lib.attention_packed_workspace(sum(lq), sum(lk), len(lq), heads, kv, hd, DEV) is not None
    run(duo_lib, lq, lk, heads, kv, hd)
    run(duo_lib, lq, lk, heads, kv, hd, scale=-0.2, pad=8)


@pytest.mark.parametrize("hd", [64, 128])
def test_split_unseen_and_infinite(duo_lib, hd):
    """Parts that see nothing, and numbers that are not finite: unseen ones have no
    influence, a seen one has, whichever part holds it."""
    say("split, numbers that are not finite", hd)
    heads, kv, lq, lk = 4, 2, 6, 3000
    Q, K, V = bf((lq, heads * hd), 1), bf((lk, kv * hd), 2), bf((lk, kv * hd), 3)
    clean = [f64(t) for t in (Q, K, V)]
    V[lk - 1], K[lk - 2] = float("nan"), float("inf")   # seen by the last query, and by the last two
    V[700, 5] = float("inf")                            # seen by all: channel 5 of the first group
    V[800, hd] = float("nan")
    dev = [t.to(DEV) for t in (Q, K, V)]
    ws = duo_lib.attention_packed_workspace(lq, lk, 1, heads, kv, hd, DEV)
    ws.fill_(255)
    O = f64(duo_lib.duo_attention_packed(*dev, cu([lq]).to(DEV), heads, kv, hd, cu_k=cu([lk]).to(DEV), ws=ws)).reshape(lq, heads, hd)
    ref, tol = S.attend(clean[0].reshape(lq, heads, hd), clean[1].reshape(lk, kv, hd), clean[2].reshape(lk, kv, hd), hd ** -0.5,
                        S.causal(lq, lk))
    assert not np.isfinite(O[4:]).any()
    assert (O[:4, :2, 5] == np.inf).all() and np.isnan(O[:4, 2:, 0]).all()
    ok = np.ones((4, heads, hd), dtype=bool)
    ok[:, :2, 5] = ok[:, 2:, 0] = False
    assert (np.abs(O[:4] - ref[:4]) <= tol[:4])[ok].all()


@pytest.mark.parametrize("hd", [64, 128])
def test_strides_and_scale(duo_lib, hd):
    say("strides, scale", hd)
    run(duo_lib, [100, 33], None, 4, 2, hd, scale=0.3, pad=8)
    run(duo_lib, [100, 33], None, 4, 2, hd, scale=-0.05, pad=16)
    run(duo_lib, [60], None, 2, 2, hd, scale=0.0)


@pytest.mark.parametrize("hd", [64, 128])
def test_many_and_long(duo_lib, hd):
    say("many workgroups", hd)
    run(duo_lib, [700, 3, 1025, 250, 64, 64, 1], None, 32, 8, hd)
    run(duo_lib, [300], [2100], 16, 2, hd)


@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("q_scale", [30.0, 400.0])
def test_large_scores(duo_lib, q_scale, hd):
    """The score's own fp32 error (in the bound) decides near-ties here."""
    say("large scores", q_scale, hd)
    run(duo_lib, [200, 31], None, 4, 2, hd, q_scale=q_scale)


def test_rising_scores(duo_lib):
    """Keys whose scores rise along the sequence: the running maximum moves in
    every block; and fall: it never does."""
    say("rising and falling scores")
    L, hd = 700, 128
    for sign in (1.0, -1.0):
        Q, V = torch.ones((L, hd)).bfloat16(), bf((L, hd), 5)
        K = (torch.arange(L)[:, None] * 0.05 * sign * torch.ones((1, hd)) / hd ** 0.5).bfloat16()
        O = duo_lib.duo_attention_packed(Q.to(DEV), K.to(DEV), V.to(DEV), cu([L]).to(DEV), 1, 1, hd)
        check(f64(O), f64(Q), f64(K), f64(V), [L], [L], 1, 1, hd)


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), float("-inf"), 3e38])
@pytest.mark.parametrize("hd", [64, 128])
def test_unseen_values_do_not_matter(duo_lib, bad, hd):
    """Rows of K and V that a query does not see, in its own sequence (later ones)
    and in the neighbours', hold anything."""
    say("unseen values", bad, hd)
    heads, kv, lq, lk = 4, 2, [40, 200, 65], [100, 200, 90]
    Q, K, V = bf((sum(lq), heads * hd), 1), bf((sum(lk), kv * hd), 2), bf((sum(lk), kv * hd), 3)
    clean = [f64(t) for t in (Q, K, V)]
    # sequence 1 from its key 70 on, all of sequence 0's V and one row of sequence 2's K
    K[100 + 70:300], V[100 + 70:300] = bad, bad
    V[:100], K[300 + 89] = bad, bad
    O = f64(duo_lib.duo_attention_packed(Q.to(DEV), K.to(DEV), V.to(DEV), cu(lq).to(DEV), heads, kv, hd,
                                         cu_k=cu(lk).to(DEV)))
    ref, tol = S.attend(*(clean[i][40 * (i == 0) + 100 * (i > 0):][:70].reshape(70, -1, hd) for i in range(3)), hd ** -0.5,
                        S.causal(70, 70))
    assert (np.abs(O[40:110].reshape(70, heads, hd) - ref) <= tol).all()
    # sequence 2: its last key is seen by its last query alone
    q, k, v = clean[0][240:304], clean[1][300:389], clean[2][300:389]
    ref, tol = S.attend(q.reshape(64, heads, hd), k.reshape(89, kv, hd), v.reshape(89, kv, hd), hd ** -0.5, S.causal(64, 89))
    assert (np.abs(O[240:304].reshape(64, heads, hd) - ref) <= tol).all()
    if not abs(bad) < float("inf"):
        # who sees such a value has it: NaN, or an infinity of its sign
        seen = O[110:240]
        assert not np.isfinite(seen).any()
        assert not np.isfinite(O[:40]).any()


def test_infinite_scores(duo_lib):
    """-inf scores weigh nothing, a row of nothing but -inf or with +inf is NaN."""
    say("infinite scores")
    L, hd = 150, 64
    Q, K, V = bf((L, hd), 1), bf((L, hd), 2), bf((L, hd), 3)
    Q[:, 0] = 1.0
    Q[100:, 0] = -1.0
    K[70, 0] = float("-inf")
    K[0, 0] = float("-inf")
    O = f64(duo_lib.duo_attention_packed(Q.to(DEV), K.to(DEV), V.to(DEV), cu([L]).to(DEV), 1, 1, hd))
    assert np.isnan(O[0]).all() and np.isnan(O[100:]).all()
    seen = S.causal(L, L)
    seen[:, [0, 70]] = False
    k = f64(K)
    k[[0, 70]] = 0.0
    ref, tol = S.attend(f64(Q)[:, None], k[:, None], f64(V)[:, None], hd ** -0.5, seen)
    assert (np.abs(O[1:100] - ref[1:100, 0]) <= tol[1:100, 0]).all()


def test_rows_in_no_sequence(duo_lib):
    """Offsets that start late and end early leave the other rows alone; ones that
    run backwards or past the end are cut."""
    say("rows in no sequence")
    heads, kv, hd, T = 2, 1, 64, 100
    Q, K, V = bf((T, heads * hd), 1), bf((T, kv * hd), 2), bf((T, kv * hd), 3)
    dev = [t.to(DEV) for t in (Q, K, V)]
    out = torch.full((T, heads * hd), 9.0, dtype=torch.bfloat16, device=DEV)
    duo_lib.duo_attention_packed(*dev, cu([30, 20], first=10).to(DEV), heads, kv, hd, out=out)
    O = f64(out)
    assert (O[:10] == 9).all() and (O[60:] == 9).all()
    check(O, f64(Q), f64(K), f64(V), [30, 20], [30, 20], heads, kv, hd, q0=10, k0=10)
    out.fill_(9.0)
    odd = torch.tensor([-5, 40, 30, 70, 1000], dtype=torch.int32, device=DEV)  # 0..40, none, 30..70, 70..100
    duo_lib.duo_attention_packed(*dev, odd, heads, kv, hd, out=out)
    check(f64(out)[70:], f64(Q)[70:], f64(K)[70:], f64(V)[70:], [30], [30], heads, kv, hd)
    assert torch.isfinite(out).all()


def test_agrees_with_attention(duo_lib):
    """Equally long sequences with as many K/V heads: the harness' attention."""
    say("against duo_attention")
    nseq, L, heads, hd = 3, 200, 4, 128
    Q, K, V = (bf((nseq * L, heads * hd), s) for s in (1, 2, 3))
    dev = [t.to(DEV) for t in (Q, K, V)]
    a = f64(duo_lib.duo_attention(*dev, nseq, L, heads, hd))
    b = f64(duo_lib.duo_attention_packed(*dev, cu([L] * nseq).to(DEV), heads, heads, hd))
    for s in range(nseq):
        r = slice(s * L, (s + 1) * L)
        _, tol = S.attend(*(f64(t)[r].reshape(L, heads, hd) for t in (Q, K, V)), hd ** -0.5, S.causal(L, L))
        assert (np.abs(a[r] - b[r]).reshape(L, heads, hd) <= 2 * tol).all()


def test_repeats_and_streams(duo_lib):
    """The same bits again, also from a stream of its own and from a replayed graph."""
    say("repeats, streams, graph")
    heads, kv, hd, lq = 8, 2, 128, [300, 77, 500]
    Q, K, V = (bf((sum(lq), n * hd), s).to(DEV) for n, s in ((heads, 1), (kv, 2), (kv, 3)))
    c = cu(lq).to(DEV)
    a = duo_lib.duo_attention_packed(Q, K, V, c, heads, kv, hd)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        b = duo_lib.duo_attention_packed(Q, K, V, c, heads, kv, hd)
    s.synchronize()
    assert torch.equal(a, b)
    out = torch.empty_like(a)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        duo_lib.duo_attention_packed(Q, K, V, c, heads, kv, hd, out=out)
    for _ in range(3):
        out.zero_()
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(a, out)


def test_refusals(duo_lib):
    say("refusals")
    Q, K, V = (bf((20, 128), s).to(DEV) for s in (1, 2, 3))
    c = cu([20]).to(DEV)
    ok = lambda **k: duo_lib.duo_attention_packed(**{**dict(Q=Q, K=K, V=V, cu_q=c, heads=2, kv_heads=2, head_dim=64), **k})
    ok()
    with pytest.raises(TypeError):
        ok(Q=Q.float())
    with pytest.raises(TypeError):
        ok(cu_q=c.long())
    with pytest.raises(ValueError):
        ok(cu_k=cu([10, 10]).to(DEV))
    with pytest.raises(ValueError):
        ok(heads=4)
    with pytest.raises(ValueError):
        ok(K=K[:, :64])
    with pytest.raises(ValueError):
        ok(V=V[:10])
    with pytest.raises(ValueError):
        ok(Q=Q.cpu())
    with pytest.raises(duo_lib.DuoError):
        ok(K=K[:10], V=V[:10])               # no cu_k, but fewer keys
    with pytest.raises(duo_lib.DuoError):
        ok(scale=float("nan"))
    with pytest.raises(duo_lib.DuoError):
        ok(head_dim=32, heads=4, kv_heads=4)
    wide = torch.zeros((20, 136), dtype=torch.bfloat16, device=DEV)
    with pytest.raises(duo_lib.DuoError):
        ok(K=wide[:, 4:132])                 # not 16-byte aligned

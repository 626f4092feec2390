"""A decoder block with norms of its query and key heads and with a window and sinks, served
step by step over a paged cache, against the float64 reference of the whole sequences; pages
that the window has left behind are taken away.

The bars are those of the other served blocks (test_serve_block_gpu.py), twice the one for
elements: there a head of queries or keys has a length of 0.05 sqrt(256) 8 = 6.4, here of
8 exp(0.3^2) = 8.75 (a norm of 8 and gains exp(0.3 n)), so that scores, and with them what roundings of
queries and keys do to the exponentials, are (8.75 / 6.4)^2 = 1.87 times as large."""

import numpy as np
import pytest
import torch

from oracle import block_ref as BR
from oracle import serve_ref as S
from test_serve_block_gpu import D, DEV, EPS, HD, HEADS, KV, THETA, f64, hidden, say, weights

pytestmark = pytest.mark.gpu
PAGE = 16


def gains(seed):
    return torch.exp(0.3 * torch.randn(HD, generator=torch.Generator().manual_seed(seed)))


def reference(h, W, fmt, window, sinks, normed):
    lin = lambda x, nm, res=None: BR.linear(x, f64(W[nm]), res)
    h, n = f64(h), len(h)
    x = BR.rmsnorm(h, EPS)
    pos = np.arange(n)

    def turned(y, heads, gain):
        if normed:
            y = S.head_norm(y, heads, HD, f64(gain), EPS)
        return BR.bf16(S.rope_at(y, heads, HD, pos, THETA)).reshape(n, heads, HD)

    q, k = turned(lin(x, "q"), HEADS, W.get("q_norm")), turned(lin(x, "k"), KV, W.get("k_norm"))
    v = lin(x, "v").reshape(n, KV, HD)
    if fmt != "bf16":
        k, v = (S.numbers(*S.quantize(t, fmt)) for t in (k, v))
    see = S.causal(n, n)
    if window:
        i, j = np.arange(n)[:, None], np.arange(n)[None, :]
        see = see & ((j > i - window) | (j < sinks))
    a = BR.bf16(S.attend(q, k, v, HD ** -0.5, see)[0]).reshape(n, HEADS * HD)
    h2 = lin(a, "o", h)
    x2 = BR.rmsnorm(h2, EPS)
    return lin(BR.silu_mul(lin(x2, "gate"), lin(x2, "up")), "down", h2)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("fmt,window,sinks", [("bf16", None, 0), ("bf16", 20, 3), ("int8", None, 0), ("int8", 33, 0), ("int4", 20, 3)])
def test_steps(duo_lib, fmt, window, sinks, dtype):
    from paper_2506_20194_amd import serve

    say("served block with norms", fmt, window, sinks, dtype)
    cuts = [[70, 20, 5, 0], [1, 1, 1, 1], [0, 33, 1, 9], [12, 1, 0, 3], [1, 1, 1, 1], [1, 1, 1, 1]]
    lens = [sum(c[i] for c in cuts) for i in range(4)]
    W = weights(11)
    W["q_norm"], W["k_norm"] = gains(1).to(dtype), gains(2).to(dtype)
    hs = hidden(lens, 12)
    Wd = {k: w.to(DEV) for k, w in W.items()}
    cfg = dict(heads=HEADS, theta=THETA, eps=EPS, window=window, sinks=sinks)
    most = -(-max(lens) // PAGE)
    order = torch.randperm(4 * most + 2, generator=torch.Generator().manual_seed(3))[:4 * most].view(4, most).int()
    cache = duo_lib.KVCache.empty(4 * most + 2, PAGE, KV, HD, fmt, DEV)
    cache.data.fill_(255)
    before, out = [0] * 4, [[] for _ in hs]
    for cut in cuts:
        table = order.clone()
        if window:  # pages whose tokens no query of this step or of a later one sees
            for s, b in enumerate(before):
                for t in range(most):
                    if (t + 1) * PAGE <= b - window + 1 and t * PAGE >= sinks:
                        table[s, t] = -1
        step = serve.Step(cache, table.to(DEV), before, cut)
        x = torch.cat([h[b:b + n] for h, b, n in zip(hs, before, cut)]).to(DEV)
        for i, part in enumerate(serve.run_block(x, Wd, cfg, cache, step).split(cut)):
            out[i].append(part)
        before = [b + n for b, n in zip(before, cut)]
    for h, o in zip(hs, out):
        y, ref = f64(torch.cat(o)), reference(h, W, fmt, window, sinks, True)
        if fmt == "bf16":
            tol = 2 * (8 * 2.0 ** -7 * np.abs(ref) + 2.0 ** -8 * np.sqrt(np.mean(ref * ref)))
            assert (np.abs(y - ref) <= tol).all(), float(np.max(np.abs(y - ref) / tol))
        else:
            assert np.linalg.norm(y - ref) < 2.0 ** -6 * np.linalg.norm(ref)


@pytest.mark.parametrize("fmt", ["int8", "bf16"])
def test_many_rows_of_a_quantised_cache(duo_lib, fmt, monkeypatch):
    """Chunks on either side of the number of rows that decides between codes and rows read
    back give the same block, up to what the rows' rounding to bf16 does."""
    from paper_2506_20194_amd import serve

    say("served block, codes and rows read back")
    W = {k: w.to(DEV) for k, w in weights(13).items()}
    cfg = dict(heads=HEADS, theta=THETA, eps=EPS)
    hs = torch.cat(hidden([300], 14)).to(DEV)
    out = []
    for many in (260 * HEADS // KV, 1 << 40):
        cache = duo_lib.KVCache.empty(32, PAGE, KV, HD, fmt, DEV)
        table = torch.arange(32, dtype=torch.int32, device=DEV)[None].contiguous()
        monkeypatch.setattr(serve, "MANY_ROWS", many)
        monkeypatch.setattr(serve, "MANY_ROWS_16", many)
        serve.run_block(hs[:40], W, cfg, cache, serve.Step(cache, table, [0], [40]))
        out.append(serve.run_block(hs[40:], W, cfg, cache, serve.Step(cache, table, [40], [260])))
    a, b = (f64(o) for o in out)
    assert np.linalg.norm(a - b) < 2.0 ** -6 * np.linalg.norm(b)

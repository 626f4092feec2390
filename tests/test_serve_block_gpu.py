"""A decoder block served step by step (prompts, chunks, single tokens) over a paged
cache, against the float64 reference of the whole sequences.  Both sides round
activations to bf16 after every operation; each stage inherits the differences of
the earlier ones, so the block's output is held to the harness' bar for its last
stage (8 units of bf16 plus 2^-8 of the root mean square) where nothing is selected
or quantised, and to 2^-6 in relative Frobenius norm where a threshold may swap an
entry or a code (the harness' bar for its streams)."""

import numpy as np
import pytest
import torch

from oracle import block_ref as BR
from oracle import duo_ref as R
from oracle import serve_ref as S

pytestmark = pytest.mark.gpu
DEV = torch.device("cuda:0")
D, FFN, HEADS, KV, HD, THETA, EPS = 256, 352, 8, 2, 64, 1e4, 1e-5
CFG = dict(heads=HEADS, theta=THETA, eps=EPS)


def say(*a):
    print("[case]", *a, flush=True)


def f64(t):
    return t.detach().cpu().double().numpy()


def weights(seed=0):
    g = torch.Generator().manual_seed(seed)
    n = dict(q=(HEADS * HD, D), k=(KV * HD, D), v=(KV * HD, D), o=(D, HEADS * HD), gate=(FFN, D), up=(FFN, D), down=(D, FFN))
    return {k: (torch.randn(s, generator=g) * 0.05).bfloat16() for k, s in n.items()}


def hidden(lens, seed=1):
    g = torch.Generator().manual_seed(seed)
    return [(torch.randn((n, D), generator=g) * torch.exp(0.5 * torch.randn(D, generator=g))).bfloat16() for n in lens]


def reference(h, W, p_x, fmt):
    """One whole sequence through the block."""
    W = {k: f64(w) for k, w in W.items()}
    lin = lambda x, nm, res=None: BR.linear(R.sparsify_tokens(x, p_x)[0] if p_x else x, W[nm], res)
    h, n = f64(h), len(h)
    x = BR.rmsnorm(h, EPS)
    pos = np.arange(n)
    q = BR.bf16(S.rope_at(lin(x, "q"), HEADS, HD, pos, THETA)).reshape(n, HEADS, HD)
    k = BR.bf16(S.rope_at(lin(x, "k"), KV, HD, pos, THETA)).reshape(n, KV, HD)
    v = lin(x, "v").reshape(n, KV, HD)
    if fmt != "bf16":
        k, v = (S.numbers(*S.quantize(t, fmt)) for t in (k, v))
    a = BR.bf16(S.attend(q, k, v, HD ** -0.5, S.causal(n, n))[0]).reshape(n, HEADS * HD)
    h2 = lin(a, "o", h)
    x2 = BR.rmsnorm(h2, EPS)
    return lin(BR.silu_mul(lin(x2, "gate"), lin(x2, "up")), "down", h2)


def served(duo, hs, W, p_x, fmt, cuts, page=16, compressed=None):
    """Every sequence through the steps of `cuts` (tokens per sequence and step)."""
    from paper_2506_20194_amd import serve

    Wd = {k: w.to(DEV) for k, w in W.items()}
    most = -(-max(len(h) for h in hs) // page)
    order = torch.randperm(len(hs) * most + 2, generator=torch.Generator().manual_seed(3))[:len(hs) * most]
    table = order.view(len(hs), most).int().to(DEV)
    cache = duo.KVCache.empty(len(hs) * most + 2, page, KV, HD, fmt, DEV)
    cache.data.fill_(255)  # NaN
    before, out = [0] * len(hs), [[] for _ in hs]
    for cut in cuts:
        step = serve.Step(cache, table, before, cut)
        x = torch.cat([h[b:b + n] for h, b, n in zip(hs, before, cut)]).to(DEV)
        y = serve.run_block(x, compressed if step.single and compressed else Wd, CFG, cache, step, p_x)
        for i, part in enumerate(y.split(cut)):
            out[i].append(part)
        before = [b + n for b, n in zip(before, cut)]
    return [f64(torch.cat(o)) for o in out]


CUTS = {
    "whole prompts": [[70, 33, 5]],
    "chunks": [[40, 20, 5], [0, 13, 0], [30, 0, 0]],
    "prompts and single tokens": [[66, 29, 1]] + [[1, 1, 1]] * 4,
    "single tokens from the start": [[1, 1, 1]] * 5,
}


@pytest.mark.parametrize("name", CUTS)
def test_steps(duo_lib, name):
    say("served block", name)
    cuts = CUTS[name]
    lens = [sum(c[i] for c in cuts) for i in range(3)]
    W, hs = weights(), hidden(lens)
    for h, y in zip(hs, served(duo_lib, hs, W, None, "bf16", cuts)):
        ref = reference(h, W, None, "bf16")
        tol = 8 * 2.0 ** -7 * np.abs(ref) + 2.0 ** -8 * np.sqrt(np.mean(ref * ref))
        assert (np.abs(y - ref) <= tol).all(), float(np.max(np.abs(y - ref) / tol))


@pytest.mark.parametrize("fmt,p_x", [("bf16", 0.5), ("int8", None), ("int8", 0.5), ("int4", None)])
def test_quantised_and_sparse(duo_lib, fmt, p_x):
    say("served block", fmt, p_x)
    cuts = [[40, 20, 5], [26, 9, 1]] + [[1, 1, 1]] * 4
    lens = [sum(c[i] for c in cuts) for i in range(3)]
    W, hs = weights(), hidden(lens)
    for h, y in zip(hs, served(duo_lib, hs, W, p_x, fmt, cuts)):
        ref = reference(h, W, p_x, fmt)
        rel = np.linalg.norm(y - ref) / np.linalg.norm(ref)
        say(f"relative Frobenius {rel:.1e}")
        assert rel < 2.0 ** -6


def test_compressed_columns(duo_lib):
    """Single tokens through the compressed columns of pruned layers give what the
    dense pruned matrices give."""
    say("served block, compressed columns")
    duo = duo_lib
    W = weights(5)
    g = torch.Generator().manual_seed(6)
    comp = {}
    for k, w in W.items():
        keep = torch.rand(w.shape, generator=g) < 0.5
        W[k] = torch.where(keep, w, torch.zeros_like(w))
        pad = torch.nn.functional.pad(keep, (0, -w.shape[1] % 32)).view(w.shape[0], -1, 32).long()
        words = (pad << torch.arange(32)).sum(-1)
        words = torch.where(words >= 2 ** 31, words - 2 ** 32, words).int()
        comp[k] = duo.dsc_compress(W[k].to(DEV), words.contiguous().to(DEV))
    cuts = [[1, 1]] * 6
    hs = hidden([6, 6], 7)
    a = served(duo, hs, W, 0.5, "int8", cuts)
    b = served(duo, hs, W, 0.5, "int8", cuts, compressed=comp)
    for x, y in zip(a, b):
        assert np.linalg.norm(x - y) < 2.0 ** -6 * np.linalg.norm(x)


def test_step_refusals(duo_lib):
    from paper_2506_20194_amd import serve

    say("step refusals")
    cache = duo_lib.KVCache.empty(4, 16, KV, HD, "bf16", DEV)
    table = torch.tensor([[0, 1], [2, 3]], dtype=torch.int32, device=DEV)
    serve.Step(cache, table, [0, 3], [32, 29])
    for before, new in (([0], [1]), ([0, 0], [33, 1]), ([30, 0], [3, 1]), ([0, -1], [1, 1])):
        with pytest.raises(ValueError):
            serve.Step(cache, table, before, new)
    step = serve.Step(cache, table, [0, 0], [3, 1])
    with pytest.raises(ValueError):
        serve.run_block(torch.zeros((3, D), dtype=torch.bfloat16, device=DEV), {}, CFG, cache, step)
    step = serve.Step(cache, table, [0, 0], [0, 0])
    assert serve.run_block(torch.zeros((0, D), dtype=torch.bfloat16, device=DEV), {}, CFG, cache, step).shape == (0, D)

"""Paged attention at a sequence's end on the GPU: what its last token holds is a
number like any other, whether the token ends a tile or not."""

import numpy as np
import pytest
import torch

from test_paged_gpu import DEV, bf, check, f64, filled, say

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("heads,kv,page,copies", [(4, 2, 16, 1), (24, 1, 64, 1), (8, 8, 256, 40)])
def test_infinite_values_in_the_last_token(duo_lib, heads, kv, page, copies, hd):
    """An infinite value gives its channel that infinity for every head of the group (all
    probabilities are positive), and changes nothing else: at ends within a tile, at its
    end, in one tile, several and split rows, and (40 copies) in rows that a wave does alone."""
    say("infinite value in the last token", heads, kv, hd, page, copies)
    lens = [1, 17, 31, 32, 33, 64, 100, 127, 700, 3001] if copies == 1 else [1, 15, 31, 32, 33, 70, 100, 127] * copies
    cache, table, K, V = filled(duo_lib, lens, kv, hd, page, "bf16", k_scale=0.2)
    v, last = V.clone(), np.cumsum(lens) - 1
    up, down = 5, hd - 1
    v[last, up], v[last, (kv - 1) * hd + down] = float("inf"), float("-inf")
    seq = torch.repeat_interleave(torch.arange(len(lens)), torch.tensor(lens))
    pos = torch.cat([torch.arange(n) for n in lens])
    duo_lib.duo_kv_write(cache, K.to(DEV), v.to(DEV), cache.slots(table.cpu(), seq, pos).to(DEV))
    Q = bf((len(lens), heads * hd), 3, 0.2)
    n = torch.tensor(lens, dtype=torch.int32, device=DEV)
    O = duo_lib.duo_attention_paged(Q.to(DEV), cache, table, n, heads).view(len(lens), heads, hd)
    G = heads // kv
    assert (O[:, :G, up] == float("inf")).all()
    assert (O[:, (kv - 1) * G:, down] == float("-inf")).all()
    # the other channels: those of finite values, which have the result of V without the infinities
    finite = O.clone()
    clean = duo_clean(duo_lib, cache, table, K, V, seq, pos, Q, n, heads).view_as(O)
    finite[:, :G, up], finite[:, (kv - 1) * G:, down] = clean[:, :G, up], clean[:, (kv - 1) * G:, down]
    assert torch.equal(finite, clean)
    some = range(len(lens)) if copies == 1 else range(8)
    rows = torch.cat([torch.arange(last[i] + 1 - lens[i], last[i] + 1) for i in some])
    check(clean[list(some)].flatten(1), Q[list(some)], K[rows], V[rows], [lens[i] for i in some], heads, kv, hd, "bf16")


def duo_clean(duo, cache, table, K, V, seq, pos, Q, n, heads):
    duo.duo_kv_write(cache, K.to(DEV), V.to(DEV), cache.slots(table.cpu(), seq, pos).to(DEV))
    return duo.duo_attention_paged(Q.to(DEV), cache, table, n, heads)


def test_infinite_values_agree_with_packed(duo_lib):
    """The packed attention of one query per sequence over the same tokens."""
    say("infinite values, paged against packed")
    lens, heads, kv, hd = [1, 20, 90, 333], 4, 2, 64
    cache, table, K, V = filled(duo_lib, lens, kv, hd, 16, "bf16", k_scale=0.2)
    v, last = V.clone(), np.cumsum(lens) - 1
    v[last, 3] = float("inf")
    v[last[1:] - 1, 70] = float("-inf")
    seq = torch.repeat_interleave(torch.arange(4), torch.tensor(lens))
    pos = torch.cat([torch.arange(n) for n in lens])
    duo_lib.duo_kv_write(cache, K.to(DEV), v.to(DEV), cache.slots(table.cpu(), seq, pos).to(DEV))
    Q = bf((4, heads * hd), 3, 0.2).to(DEV)
    a = duo_lib.duo_attention_paged(Q, cache, table, torch.tensor(lens, dtype=torch.int32, device=DEV), heads)
    cu_q = torch.arange(5, dtype=torch.int32, device=DEV)
    cu_k = torch.tensor(np.concatenate(([0], np.cumsum(lens))), dtype=torch.int32, device=DEV)
    b = duo_lib.duo_attention_packed(Q, K.to(DEV), v.to(DEV), cu_q, heads, kv, hd, cu_k=cu_k)
    a, b = f64(a), f64(b)
    assert not np.isnan(a).any()
    assert (np.isinf(a) == np.isinf(b)).all() and (a[np.isinf(a)] == b[np.isinf(a)]).all()

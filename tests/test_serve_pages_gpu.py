"""A page that is not in the cache, in the steps of a served block: the sequence
that needs it is NaN, by chunks as by single tokens, and the others are as they are
without it."""

import pytest
import torch

from test_serve_block_gpu import CFG, D, DEV, HD, KV, hidden, say, weights

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("fmt", ["bf16", "int8", "int4"])
@pytest.mark.parametrize("bad", [-1, 8, 2 ** 31 - 1])
@pytest.mark.parametrize("before,new", [([0, 0, 0], [40, 5, 20]), ([0, 0, 0], [33, 1, 1]), ([36, 4, 3], [3, 2, 18]),
                                        ([36, 4, 3], [1, 0, 1]), ([36, 4, 3], [1, 1, 1])])
def test_page_outside(duo_lib, fmt, bad, before, new):
    """Sequence 0 lacks its third page, sequence 2 has a page that it does not need and
    that is not there either."""
    from paper_2506_20194_amd import serve

    say("served page outside", fmt, bad, before, new)
    W = {k: w.to(DEV) for k, w in weights().items()}
    out = []
    for third in (2, bad):
        cache = duo_lib.KVCache.empty(8, 16, KV, HD, fmt, DEV)
        cache.data.zero_()
        good = torch.tensor([[0, 1, 2], [3, 4, 7], [5, 6, 7]], dtype=torch.int32, device=DEV)
        if any(before):
            x = torch.cat(hidden(before, 3)).to(DEV)
            serve.run_block(x, W, CFG, cache, serve.Step(cache, good, [0, 0, 0], before))
        table = good.clone()
        table[0, 2] = third
        table[2, 2] = 7 if third == 2 else bad
        x = torch.cat(hidden(new, 4)).to(DEV)
        y = serve.run_block(x, W, CFG, cache, serve.Step(cache, table, before, new))
        out.append(y.split(new))
    (a0, *a), (b0, *b) = out
    assert torch.isfinite(torch.cat((a0, *a))).all()
    assert torch.isnan(b0).all() and b0.shape == (new[0], D)
    for x, y in zip(a, b):
        assert torch.equal(x, y)

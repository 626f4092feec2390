"""A served step whose first block is captured into a graph: everything that the block needs is the
step's from its start on.  Replays, with eager work between them, give the eager result."""

import pytest
import torch

from test_serve_block_gpu import CFG, DEV, HD, KV, hidden, say, weights

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("many", [0, 1 << 40], ids=["rows read back", "pages"])
@pytest.mark.parametrize("fmt", ["bf16", "int8"])
def test_first_block_in_a_graph(duo_lib, fmt, many, monkeypatch):
    from paper_2506_20194_amd import serve

    say("served step in a graph", fmt, many)
    monkeypatch.setattr(serve, "MANY_ROWS", many)
    monkeypatch.setattr(serve, "MANY_ROWS_16", many)
    W = {k: w.to(DEV) for k, w in weights(5).items()}
    cache = duo_lib.KVCache.empty(40, 16, KV, HD, fmt, DEV)
    cache.data.zero_()
    table = torch.randperm(40, generator=torch.Generator().manual_seed(2))[:36].view(3, 12).int().to(DEV)
    before, new = [100, 7, 0], [60, 40, 25]
    x0, x1 = (torch.cat(hidden(n, s)).to(DEV) for n, s in ((before, 6), (new, 7)))
    serve.run_block(x0, W, CFG, cache, serve.Step(cache, table, [0] * 3, before))
    want = serve.run_block(x1, W, CFG, cache, serve.Step(cache, table, before, new))
    assert torch.isfinite(want).all()
    step = serve.Step(cache, table, before, new)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y = serve.run_block(x1, W, CFG, cache, step)
    for _ in range(3):
        y.fill_(7.0)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, want)
        serve.run_block(x1, W, CFG, cache, serve.Step(cache, table, before, new))
        torch.cuda.synchronize()

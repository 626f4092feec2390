"""Packed attention split over the keys: two launches and a workspace, and the same bits
every time."""

import pytest
import torch

from test_packed_gpu import DEV, bf, check, cu, f64, say

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("heads,kv,lq,lk", [(8, 8, [3, 40], [4097, 600]), (16, 2, [1, 20], [9000, 2]), (12, 3, [5, 1, 64], [3000, 0, 1500])])
def test_repeats_streams_and_graph(duo_lib, heads, kv, lq, lk, hd):
    """From a workspace that holds anything, from a stream of its own, and from a
    replayed graph whose offsets change, into an output that held something else."""
    say("packed split repeats, streams, graph", heads, kv, lq, lk, hd)
    duo, n = duo_lib, len(lq)
    Q, K, V = bf((sum(lq), heads * hd), 1, 1.5), bf((sum(lk), kv * hd), 2), bf((sum(lk), kv * hd), 3)
    dev = [t.to(DEV) for t in (Q, K, V)]
    a, b = cu(lq).to(DEV), cu(lk).to(DEV)
    ws = duo.attention_packed_workspace(sum(lq), sum(lk), n, heads, kv, hd, DEV)
    assert ws is not None

    def call(out=None, ws=None):
        return duo.duo_attention_packed(*dev, a, heads, kv, hd, cu_k=b, out=out, ws=ws)

    first = call()
    check(f64(first), f64(Q), f64(K), f64(V), lq, lk, heads, kv, hd)
    for fill in (0, 255):
        ws.fill_(fill)
        assert torch.equal(first, call(ws=ws))
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        other = call()
    s.synchronize()
    assert torch.equal(first, other)
    out = torch.empty_like(first)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        call(out=out, ws=ws)
    fewer = [max(x - 1, 0) for x in lq], [x // 2 for x in lk]
    for q, k in ((lq, lk), fewer, ([0] * n, lk), (lq, lk)):
        a.copy_(cu(q))
        b.copy_(cu(k))
        want = torch.full_like(out, 9.0)
        call(out=want)
        out.fill_(9.0)
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(want, out)
        assert (out[sum(q):] == 9.0).all()
        check(f64(out), f64(Q), f64(K), f64(V), q, k, heads, kv, hd)
    assert torch.equal(first, out)

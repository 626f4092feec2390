"""A single row of a matrix of any width: no stride lies between it and another one, so
none is refused."""

import pytest
import torch

pytestmark = pytest.mark.gpu
DEV = torch.device("cuda:0")


def row(w, extra, seed):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn((3, w + extra), generator=g).bfloat16().to(DEV)[:1, :w]
    assert x.stride(0) == w + extra
    return x


@pytest.mark.parametrize("extra", [1, 4, 12])
def test_single_rows(duo_lib, extra):
    print("[case] single rows", extra, flush=True)
    duo, heads, kv, hd = duo_lib, 4, 2, 64
    q, k, v = row(heads * hd, extra, 1), row(kv * hd, extra, 2), row(kv * hd, extra, 3)
    Q, K, V = (t.contiguous() for t in (q, k, v))
    pos, slot = torch.tensor([7], dtype=torch.int32, device=DEV), torch.tensor([5], device=DEV)
    o = row(heads * hd, extra, 4)
    assert torch.equal(duo.duo_rope_at(q, heads, hd, pos, out=o), duo.duo_rope_at(Q, heads, hd, pos))
    a, b = (duo.KVCache.empty(2, 16, kv, hd, "bf16", DEV) for _ in "ab")
    for c, x, y in ((a, k, v), (b, K, V)):
        c.data.zero_()
        duo.duo_kv_write(c, x, y, slot)
    assert torch.equal(a.data, b.data)
    assert all(torch.equal(x, y) for x, y in zip(duo.duo_kv_read(a, slot, out=(row(kv * hd, extra, 5), row(kv * hd, extra, 6))),
                                                 (K, V)))
    cu = torch.tensor([0, 1], dtype=torch.int32, device=DEV)
    assert torch.equal(duo.duo_attention_packed(q, k, v, cu, heads, kv, hd, out=o), duo.duo_attention_packed(Q, K, V, cu, heads, kv, hd))
    table, lens = torch.zeros((1, 1), dtype=torch.int32, device=DEV), torch.tensor([6], dtype=torch.int32, device=DEV)
    assert torch.equal(duo.duo_attention_paged(q, a, table, lens, heads, out=o), duo.duo_attention_paged(Q, a, table, lens, heads))

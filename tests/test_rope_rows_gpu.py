"""Rotation of more rows than one launch has workgroups."""

import pytest
import torch

pytestmark = pytest.mark.gpu
DEV = torch.device("cuda:0")


def test_many_rows(duo_lib):
    """2^24 + 5 rows, so that a workgroup takes two: the same bits as a few rows at a time."""
    m, heads, hd = 2 ** 24 + 5, 129, 2
    print("[case] rope_at", m, heads, hd, flush=True)
    x = torch.empty((m, heads * hd), dtype=torch.bfloat16, device=DEV)
    g = torch.Generator(device=DEV)
    g.manual_seed(1)
    for part in x.split(2 ** 20):
        part.copy_(torch.randn(part.shape, generator=g, device=DEV))
    pos = torch.randint(0, 100000, (m,), generator=g, device=DEV, dtype=torch.int32)
    some = [(0, 9), (2 ** 23 - 3, 2 ** 23 + 4), (2 ** 24 - 5, m)]
    want = [duo_lib.duo_rope_at(x[a:b], heads, hd, pos[a:b]) for a, b in some]
    duo_lib.duo_rope_at(x, heads, hd, pos, out=x)
    for (a, b), w in zip(some, want):
        assert torch.equal(x[a:b], w)

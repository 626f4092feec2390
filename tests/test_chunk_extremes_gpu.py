"""Attention of new tokens over the cache where finite numbers lie very far apart: values, keys
and queries of 2^100 and 2^-100 beside ordinary ones, seen by all queries, by some of them or by
none, in sequences of few rows, of many and of more than have their numbers made before.  The
reference and its bounds are those of test_chunk_gpu.py."""

import numpy as np
import pytest
import torch

from oracle import serve_ref as S
from test_chunk_gpu import FMTS, Batch, say, seen

pytestmark = pytest.mark.gpu
ROWS = [(2, 9), (16, 60), (16, 150), (16, 170)]  # heads (on 2) and new tokens: 9, 480, 1200 and 1360 rows


def scaled(t, rows, power):
    t[rows] = (t[rows].float() * 2.0 ** power).bfloat16()


@pytest.mark.parametrize("power", [100, -100])
@pytest.mark.parametrize("where", ["values", "keys"])
@pytest.mark.parametrize("heads,lq", ROWS)
@pytest.mark.parametrize("fmt", FMTS)
def test_unseen_behind(duo_lib, fmt, heads, lq, where, power):
    """Prompts whose first tile holds a number that the queries before it do not see.  A key of 2^100
    makes scores that fp32 cannot tell apart (neighbours above 2^24 are 2 apart, factors of e^2
    of a probability): with it only the queries that do not see it are compared."""
    say("chunk extremes, unseen behind", fmt, heads, lq, where, power)
    at = min(40, lq - 2)

    def touch(b):
        for s in range(2):
            scaled(b.V if where == "values" else b.K, [lq * s + at], power)

    b = Batch(duo_lib, [(lq, lq), (lq, lq)], heads, 2, 128, 16, fmt, touch=touch)
    O = b.run()
    if where == "keys" and power > 0:
        first = [t.view(2, lq, -1)[:, :at].flatten(0, 1) for t in (b.K, b.V, b.Q, O)]
        b.seqs, (b.K, b.V, b.Q, O) = [(at, at)] * 2, first
    b.check(O)


@pytest.mark.parametrize("power", [100, -100])
@pytest.mark.parametrize("heads,lq", ROWS)
@pytest.mark.parametrize("fmt", FMTS)
def test_unseen_before(duo_lib, fmt, heads, lq, power):
    """The first tile of a window holds numbers that no query sees, or the first ones alone."""
    say("chunk extremes, before the window", fmt, heads, lq, power)
    n, window = 700, 100
    first = n - lq - window + 1  # the first that is seen

    def touch(b):
        scaled(b.V, [first - 1, first - 2, first + 2], power)
        scaled(b.K, [first - 1], power)

    b = Batch(duo_lib, [(lq, n), (lq, 90)], heads, 2, 128, 64, fmt, window=window, sinks=3, touch=touch)
    b.check(b.run())


@pytest.mark.parametrize("power", [100, -100])
@pytest.mark.parametrize("heads,lq", ROWS)
@pytest.mark.parametrize("fmt", FMTS)
def test_page_of_another(duo_lib, fmt, heads, lq, power):
    """A page that is not there, in the first tile and behind the window: whatever page 0 holds,
    queries that do not see it get the same bits."""
    say("chunk extremes, page 0", fmt, heads, lq, power)
    n, window = 300, 100
    out = []
    for p in (0, power):
        b = Batch(duo_lib, [(lq, n)], heads, 2, 128, 16, fmt, window=window, sinks=0)
        page = (n - lq - window + 1) // 16  # the first that some query sees
        free = next(i for i in range(len(b.cache.data)) if not (b.table == i).any())
        b.cache.data[free] = b.cache.data[0]
        b.table[b.table == 0] = free
        v = torch.randn((16, 2 * 128), generator=torch.Generator().manual_seed(3)) * 2.0 ** p
        duo_lib.duo_kv_write(b.cache, v.bfloat16().cuda(), v.bfloat16().cuda(), torch.arange(16).cuda())
        b.table[0, page] = -1
        O = b.run()
        hit = torch.from_numpy(seen(lq, n, window, 0)[:, 16 * page:16 * page + 16].any(1)).to(O.device)
        assert torch.isnan(O[hit]).all() and torch.isfinite(O[~hit]).all()
        out.append(O[~hit])
    assert torch.equal(*out)


@pytest.mark.parametrize("power", [80, 110, -80, -110])
@pytest.mark.parametrize("at", [[90], [3, 400], [699], list(range(64)), list(range(64, 700))],
                         ids=lambda a: f"{a[0]}.{len(a)}.{a[-1]}")
@pytest.mark.parametrize("heads,lq", ROWS)
@pytest.mark.parametrize("fmt", FMTS)
def test_seen(duo_lib, fmt, heads, lq, at, power):
    """Values far from the others that all queries see, or the last ones."""
    say("chunk extremes, seen values", fmt, heads, lq, at[:4], power)
    if len(at) > 2 and power == 110:
        power = 100  # values times tokens stay in range
    b = Batch(duo_lib, [(lq, 700), (70, 70)], heads, 2, 128, 16, fmt, touch=lambda b: scaled(b.V, at, power))
    b.check(b.run())


@pytest.mark.parametrize("heads,lq", ROWS)
@pytest.mark.parametrize("fmt", FMTS)
def test_everything(duo_lib, fmt, heads, lq, monkeypatch):
    """Values of all sizes, zeros among them, keys and queries too, in parts and whole.  Some scores are
    hundreds apart here, and the tokens with the high ones may have the small values: a probability below 2^-126 of the
    largest is 0 in fp32, so that up to 2^-126 |v| of each token is missing (the sum of probabilities is at least 1)."""
    say("chunk extremes, everything", fmt, heads, lq)
    attend = S.attend

    def wider(Q, K, V, scale, see, extra=0.0):
        O, bound = attend(Q, K, V, scale, see, extra)
        lost = 2.0 ** -126 * np.einsum("ln,nhd->lhd", see.astype(float), np.abs(V))
        return O, bound + np.repeat(lost, Q.shape[1] // V.shape[1], 1)

    monkeypatch.setattr(S, "attend", wider)
    g = torch.Generator().manual_seed(21)

    def spread(x, lo, hi, some):
        e = torch.randint(lo, hi + 1, (len(x),), generator=g).float()
        e = torch.where(torch.rand(len(x), generator=g) < some, e, 0.0)
        x.copy_((x.float() * torch.exp2(e)[:, None]).bfloat16())

    def touch(b):
        spread(b.V, -110, 100, 0.3)
        b.V[torch.rand(len(b.V), generator=g) < 0.1] = 0.0
        b.V[2000:2700] = b.V[2000:2700].float().clamp(-1, 1).mul(2.0 ** -60).bfloat16()
        spread(b.K, -110, 4, 0.2)

    seqs = [(lq, 700), (lq, lq), (9, 1291), (lq, 2500)]
    b = Batch(duo_lib, seqs, heads, 2, 128, 16, fmt, touch=touch)
    spread(b.Q, -100, 5, 0.3)
    b.check(b.run())


@pytest.mark.parametrize("lq", [10, 40])
@pytest.mark.parametrize("fmt", FMTS)
def test_zeros_beside_small_values(duo_lib, fmt, lq):
    """Tokens whose values are all 0 have no part in an output, however small the others' are."""
    say("chunk extremes, zeros", fmt, lq)

    def touch(b):
        scaled(b.V, slice(0, 39), -80)
        b.V[5:39:7] = 0.0
        b.K[5:39:7] *= 2.0

    b = Batch(duo_lib, [(lq, 40)], 16, 1, 64, 16, fmt, touch=touch)
    b.check(b.run())


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("heads", [16, 17])
def test_both_sides_of_few_rows(duo_lib, fmt, heads):
    """The same data by 64 rows and by 68: one path and the other."""
    say("chunk extremes, 64 rows and 68", fmt, heads)
    for power in (80, 100, -80, -100):
        b = Batch(duo_lib, [(4, 300)], heads, 1, 128, 16, fmt, touch=lambda b: scaled(b.V, [70, 200], power))
        b.check(b.run())
        b = Batch(duo_lib, [(4, 300)], heads, 1, 128, 16, fmt, touch=lambda b: scaled(b.V, slice(0, 64), power))
        b.check(b.run())


@pytest.mark.parametrize("heads,lq", ROWS[1:])
@pytest.mark.parametrize("fmt", FMTS[1:])
def test_largest(duo_lib, fmt, heads, lq):
    """The largest numbers that there are."""
    say("chunk extremes, largest values", fmt, heads, lq)

    def touch(b):
        b.V[5] = b.V[5].sign() * torch.finfo(torch.bfloat16).max

    b = Batch(duo_lib, [(lq, 700)], heads, 2, 128, 16, fmt, touch=touch)
    b.check(b.run())


@pytest.mark.parametrize("heads,lq", ROWS[1:])
@pytest.mark.parametrize("fmt", FMTS[1:])
def test_ordinary_sizes(duo_lib, fmt, heads, lq):
    """Values of ordinary sizes (tokens' largest ones from 2^-6 to 2^5) need no powers: with all of them times a power of
    two the outputs are times that, bit for bit, as the same steps were taken."""
    say("chunk, ordinary sizes", fmt, heads, lq)

    def run(power):
        b = Batch(duo_lib, [(lq, 700), (lq, lq)], heads, 2, 128, 16, fmt, touch=lambda b: scaled(b.V, slice(None), power))
        O = b.run()
        b.check(O)
        return O.float() * 2.0 ** -power

    want = run(0)
    for power in (-5, -4, -3, -2, -1, 1, 2):
        assert torch.equal(run(power), want), power

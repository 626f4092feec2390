"""The paged key-value cache and the rotation by positions on the GPU, against the
float64 reference.  Cache bytes are compared bit for bit: x and a scale are
bfloat16, so a quotient is a tie or at least 2^-16 away from one, and every correct
rounding gives the same code.  A rotated number may be one rounding to bf16 off
(half a unit of eight bits: 2^-8 of it) plus the fp32 error of two products and a cosine (2^-22 of the pair)."""

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


def rows(m, w, seed, ld=None):
    """m x w bf16 rows of mixed sizes, a view of rows ld wide."""
    g = torch.Generator().manual_seed(seed)
    x = torch.randn((m, ld or w), generator=g) * torch.exp(2 * torch.randn((m, 1), generator=g))
    return x.bfloat16()[:, :w]


@pytest.mark.parametrize("m,heads,hd,ld,longest", [
    (1, 1, 64, 64, 10), (3, 8, 128, 1024, 100), (70, 64, 128, 8192, 1 << 20), (257, 5, 64, 328, 8192),
    (33, 2, 96, 192, 4096), (17, 3, 80, 240, 300), (9, 3, 10, 31, 50), (5, 1, 256, 256, 131072), (300, 1, 2, 2, 999),
])
def test_rope_at(duo_lib, m, heads, hd, ld, longest):
    say("rope_at", m, heads, hd, ld, longest)
    x = rows(m, heads * hd, m + hd, ld)
    pos = torch.randint(0, longest, (m,), generator=torch.Generator().manual_seed(m), dtype=torch.int32)
    pos[0] = longest - 1
    if m > 2:
        pos[1], pos[2] = 0, -7
    ref = S.rope_at(f64(x), heads, hd, pos.numpy(), 1e4)
    size = np.abs(f64(x).reshape(m, heads, 2, -1)).sum(2, keepdims=True).repeat(2, 2).reshape(m, -1)
    tol = 2.0 ** -8 * 1.02 * np.abs(ref) + 2.0 ** -22 * size + 1e-38
    xd = torch.empty((m, ld), dtype=torch.bfloat16, device=DEV)[:, :heads * hd]
    xd.copy_(x)
    y = duo_lib.duo_rope_at(xd, heads, hd, pos.to(DEV))
    assert (np.abs(f64(y) - ref) <= tol).all()
    assert torch.equal(xd.cpu(), x)
    duo_lib.duo_rope_at(xd, heads, hd, pos.to(DEV), out=xd)  # in place
    assert torch.equal(xd, y)


def test_rope_at_agrees_with_rope(duo_lib):
    """Positions 0, 1, .. of equally long sequences: the harness' rotation, up to
    one unit of bf16 where the two round their cosines apart."""
    say("rope_at against rope")
    x = rows(600, 4 * 128, 3).to(DEV)
    y = duo_lib.duo_rope_at(x, 4, 128, (torch.arange(600, device=DEV) % 300).int())
    z = duo_lib.duo_rope(x.clone(), 4, 128, 300)
    d = (y.double() - z.double()).abs()
    assert (d <= 2.0 ** -7 * z.double().abs() + 2.0 ** -20 * x.double().abs().max()).all()
    assert float((d > 0).double().mean()) < 1e-3


def _special(x):
    """Groups at the edges of the formats, in rows of at least two groups."""
    big = torch.finfo(torch.bfloat16).max
    x[0, :32] = 0.0
    x[1, :32] = -0.0
    x[2, 3] = float("nan")
    x[3, 5] = float("-inf")
    x[4, :32] = 2.0 ** -130
    x[5, :32] = torch.linspace(-2.0 ** -120, 2.0 ** -120, 32).bfloat16()  # its scale is below 2^-126 in 8 bits alone
    x[6, :32] = big
    x[7, :32] = torch.tensor([127.0] + [0.5 + i for i in range(31)]).bfloat16()  # ties with s = 1 (8 bits)
    x[8, :32] = torch.tensor([-7.0] + [(i % 14) / 2 - 3.5 for i in range(31)]).bfloat16()  # ties with s = 1 (4 bits)
    x[9, :32] = 1.0
    x[9, 31] = 3e38
    return x


@pytest.mark.parametrize("fmt", ["bf16", "int8", "int4"])
@pytest.mark.parametrize("kv,hd,page,m", [(1, 64, 16, 10), (3, 128, 64, 77), (8, 128, 16, 130), (5, 64, 256, 300),
                                          (2, 128, 32, 33), (1, 128, 128, 11)])
def test_write_and_read(duo_lib, fmt, kv, hd, page, m):
    say("write and read", fmt, kv, hd, page, m)
    g = torch.Generator().manual_seed(m)
    pages = -(-m // page) + 3
    w = kv * hd
    K, V = _special(rows(m, w, 1, w + 8)), _special(rows(m, w, 2).flip(1)).contiguous()
    slots = torch.randperm(pages * page, generator=g)[:m]
    if m > 20:
        slots[11], slots[12], slots[13] = -1, pages * page, 1 << 40
    cache = duo_lib.KVCache.empty(pages, page, kv, hd, fmt, DEV)
    before = torch.randint(0, 256, cache.data.shape, generator=g, dtype=torch.uint8)
    cache.data.copy_(before)
    Kd = torch.empty((m, w + 8), dtype=torch.bfloat16, device=DEV)[:, :w]
    Kd.copy_(K)
    duo_lib.duo_kv_write(cache, Kd, V.to(DEV), slots.to(DEV))
    bits = [x.view(m, kv, hd) for x in (K.contiguous(), V)]
    if fmt == "bf16":  # any bit pattern, NaN among them
        want = before.clone()
        for which, x in enumerate(bits):
            for t, s in enumerate(slots.tolist()):
                if 0 <= s < pages * page:
                    at = (which * page + s % page) * 2 * hd
                    want[s // page, :, at:at + 2 * hd] = x[t].contiguous().view(torch.uint8)
        want = want.numpy()
    else:
        want = S.write(before.numpy(), *(f64(x) for x in bits), slots.numpy(), page, hd, fmt)
    assert np.array_equal(cache.data.cpu().numpy(), want)
    # what is read back, in another order, with rows that are not there
    order = torch.randperm(m, generator=g)
    out = [torch.full((m, w + 16), 5.0, dtype=torch.bfloat16, device=DEV) for _ in "KV"]
    got = duo_lib.duo_kv_read(cache, slots[order].to(DEV), out=[o[:, :w] for o in out])
    for x, y, o in zip(bits, got, out):
        ref = f64(x) if fmt == "bf16" else S.numbers(*S.quantize(f64(x), fmt))
        ref = ref.reshape(m, w)[order.numpy()]
        ref[((slots[order] < 0) | (slots[order] >= pages * page)).numpy()] = 0.0
        top = float(torch.finfo(torch.bfloat16).max)
        ref = np.where(np.isfinite(ref), np.clip(S.bf16(np.where(np.isfinite(ref), ref, 0.0)), -top, top), ref)
        assert np.array_equal(f64(y), ref, equal_nan=True)
        assert (o[:, w:] == 5.0).all()


@pytest.mark.parametrize("fmt", ["int8", "int4"])
def test_error_of_a_stored_number(duo_lib, fmt):
    """A finite number comes back within half a step of its group (the scale's own
    rounding, 2^-9, may push the largest half a step further) and one rounding."""
    say("error of a stored number", fmt)
    m, kv, hd = 500, 4, 128
    K, V = rows(m, kv * hd, 4), rows(m, kv * hd, 5)
    cache = duo_lib.KVCache.empty(8, 64, kv, hd, fmt, DEV)
    slots = torch.arange(m, device=DEV)
    duo_lib.duo_kv_write(cache, K.to(DEV), V.to(DEV), slots)
    for x, y in zip((K, V), duo_lib.duo_kv_read(cache, slots)):
        x, y = f64(x).reshape(-1, 32), f64(y).reshape(-1, 32)
        step = np.abs(x).max(1, keepdims=True) / S.MOST[fmt] * (1 + 2.0 ** -8)
        assert (np.abs(x - y) <= step / 2 + 2.0 ** -8 * np.abs(x).max(1, keepdims=True)).all()


def test_nothing_to_do(duo_lib):
    say("no tokens")
    cache = duo_lib.KVCache.empty(2, 16, 2, 64, "int8", DEV)
    before = cache.data.clone()
    e = torch.empty((0, 128), dtype=torch.bfloat16, device=DEV)
    none = torch.empty(0, dtype=torch.int64, device=DEV)
    duo_lib.duo_kv_write(cache, e, e, none)
    assert [t.shape for t in duo_lib.duo_kv_read(cache, none)] == [(0, 128)] * 2
    assert duo_lib.duo_rope_at(e, 2, 64, none.int()).shape == (0, 128)
    assert torch.equal(cache.data, before)


@pytest.mark.parametrize("fmt", ["bf16", "int8", "int4"])
def test_slots_past_32_bits(duo_lib, fmt):
    """Rows whose bytes lie more than 4 GiB into the cache."""
    say("offsets past 32 bits", fmt)
    page, kv, hd = 256, 8, 128
    pages = -(-(9 << 29) // duo_lib.kv_page_bytes(page, kv, hd, fmt))
    cache = duo_lib.KVCache.empty(pages, page, kv, hd, fmt, DEV)
    K, V = rows(6, kv * hd, 6), rows(6, kv * hd, 7)
    last = pages * page - 1
    slots = torch.tensor([last, 0, last - page, last // 2, last - 1, 1])
    duo_lib.duo_kv_write(cache, K.to(DEV), V.to(DEV), slots.to(DEV))
    for x, y in zip((K, V), duo_lib.duo_kv_read(cache, slots.to(DEV))):
        x = f64(x).reshape(6, kv, hd)
        ref = x if fmt == "bf16" else S.bf16(S.numbers(*S.quantize(x, fmt)))
        assert np.array_equal(f64(y), ref.reshape(6, -1))
    tail = cache.data[-1].cpu().numpy()
    want = S.write(tail[None], *(f64(t[[0, 4]]).reshape(2, kv, hd) for t in (K, V)), np.array([page - 1, page - 2]), page,
                   hd, fmt)
    assert np.array_equal(tail, want[0])

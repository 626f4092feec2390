"""Head norms with the rotation, and keys rotated into the paged cache, on the GPU.
A normed and rotated number may be off by its rounding to bf16 (2^-8 of it), and, as parts
of the pair that it comes from, by the fp32 errors of the rotation (2^-22: two products and
a cosine), of the sum of squares (at most head_dim 2^-24, half of that in the root) and of
the root, the mean, eps and two products (16 2^-24).  What goes into the cache is compared bit
for bit with what the calls store that it stands for."""

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
    g = torch.Generator().manual_seed(seed)
    x = torch.randn((m, ld or w), generator=g) * torch.exp(2 * torch.randn((m, 1), generator=g))
    return x.bfloat16()[:, :w]


def on_gpu(x, ld):
    y = torch.empty((x.shape[0], ld), dtype=x.dtype, device=DEV)[:, :x.shape[1]]
    return y.copy_(x)


def gains(n, seed, dtype):
    return torch.exp(0.5 * torch.randn(n, generator=torch.Generator().manual_seed(seed))).to(dtype)


@pytest.mark.parametrize("dtype", [None, torch.bfloat16, torch.float32])
@pytest.mark.parametrize("m,heads,hd,ld", [
    (1, 1, 64, 64), (3, 8, 128, 1024), (70, 64, 128, 8192), (257, 5, 64, 328), (33, 2, 96, 192), (17, 3, 80, 240),
    (9, 3, 10, 31), (5, 1, 256, 256), (300, 1, 2, 2), (21, 2, 16, 40), (2, 3, 144, 435), (1, 40, 250, 10000),
])
def test_head_norm_rope(duo_lib, m, heads, hd, ld, dtype):
    say("head_norm_rope", m, heads, hd, ld, dtype)
    x = rows(m, heads * hd, m + hd, ld)
    x[0] *= 2.0 ** -20  # where eps counts
    pos = torch.randint(0, 1 << 17, (m,), generator=torch.Generator().manual_seed(m), dtype=torch.int32)
    if m > 2:
        pos[1], pos[2] = 0, -7
    gain = None if dtype is None else gains(hd, 5, dtype)
    normed = S.head_norm(f64(x), heads, hd, None if gain is None else f64(gain), 1e-5)
    ref = S.rope_at(normed, heads, hd, pos.numpy(), 1e4)
    size = np.abs(normed.reshape(m, heads, 2, -1)).sum(2, keepdims=True).repeat(2, 2).reshape(m, -1)
    tol = 2.0 ** -8 * 1.02 * np.abs(ref) + (2.0 ** -22 + (hd / 2 + 16) * 2.0 ** -24) * size + 1e-38
    xd = on_gpu(x, ld)
    g = None if gain is None else gain.to(DEV)
    y = duo_lib.duo_head_norm_rope(xd, heads, hd, pos.to(DEV), g)
    assert (np.abs(f64(y) - ref) <= tol).all()
    assert torch.equal(xd.cpu(), x)
    out = torch.full((m, heads * hd + 3), 9.0, dtype=torch.bfloat16, device=DEV)  # rows that start anywhere
    duo_lib.duo_head_norm_rope(xd, heads, hd, pos.to(DEV), g, out=out[:, :heads * hd])
    assert (out[:, heads * hd:] == 9.0).all()
    assert (np.abs(f64(out[:, :heads * hd]) - ref) <= tol).all()
    duo_lib.duo_head_norm_rope(xd, heads, hd, pos.to(DEV), g, out=xd)  # in place
    assert torch.equal(xd, y)


def test_head_norm_of_zeros_and_no_rows(duo_lib):
    say("head_norm_rope of zeros")
    x = torch.zeros((4, 256), dtype=torch.bfloat16, device=DEV)
    pos = torch.arange(4, device=DEV, dtype=torch.int32)
    assert (duo_lib.duo_head_norm_rope(x, 2, 128, pos) == 0).all()
    x[2, 5] = float("inf")
    y = duo_lib.duo_head_norm_rope(x, 2, 128, pos)
    assert torch.isnan(y[2, 5]) and (y[[0, 1, 3]] == 0).all() and (y[2, 128:] == 0).all()
    assert duo_lib.duo_head_norm_rope(x[:0], 2, 128, pos[:0]).shape == (0, 256)


@pytest.mark.parametrize("norm", [None, "ones", torch.bfloat16, torch.float32])
@pytest.mark.parametrize("fmt", ["bf16", "int8", "int4"])
@pytest.mark.parametrize("m,heads,kv,hd,page", [(1, 8, 1, 128, 16), (37, 6, 3, 64, 64), (300, 64, 8, 128, 32), (5, 0, 2, 128, 256),
                                                (1030, 4, 1, 64, 16)])
def test_append(duo_lib, m, heads, kv, hd, page, fmt, norm):
    """Bytes of the cache and rotated queries, against the calls one by one."""
    say("append", m, heads, kv, hd, page, fmt, norm)
    d = duo_lib
    K, V, Q = (rows(m, n * hd, 7 + i) for i, n in enumerate((kv, kv, max(heads, 1))))
    K[m // 2, 3] = float("nan")
    V[m // 3, 5] = float("-inf")
    K[0, :32] = 0.0
    pos = torch.randint(0, 1 << 17, (m,), generator=torch.Generator().manual_seed(m), dtype=torch.int32).to(DEV)
    pages = -(-m // page) + 3
    slots = torch.randperm(pages * page, generator=torch.Generator().manual_seed(1))[:m]
    if m > 4:
        slots[1], slots[3] = -1, pages * page  # skipped
    slots = slots.to(DEV)
    one, two = (d.KVCache(torch.full_like(d.KVCache.empty(pages, page, kv, hd, fmt, DEV).data, 77), page, kv, hd, fmt)
                for _ in range(2))
    kd, vd, qd = on_gpu(K, kv * hd + 8), on_gpu(V, kv * hd + 16), on_gpu(Q, max(heads, 1) * hd + 8)
    typed = isinstance(norm, torch.dtype)
    kg, qg = (gains(hd, s, norm).to(DEV) if typed else None for s in (1, 2))
    eps = None if norm is None else 1e-5
    if norm is None:
        k2 = d.duo_rope_at(kd, kv, hd, pos, 1e5)
        q2 = d.duo_rope_at(qd, heads, hd, pos, 1e5) if heads else None
    else:
        k2 = d.duo_head_norm_rope(kd, kv, hd, pos, kg, eps, 1e5)
        q2 = d.duo_head_norm_rope(qd, heads, hd, pos, qg, eps, 1e5) if heads else None
    d.duo_kv_write(two, k2, vd, slots)
    q1 = d.duo_kv_append(one, kd, vd, slots, pos, 1e5, eps, kg, qd if heads else None, qg if heads else None)
    assert torch.equal(one.data, two.data)
    if heads:
        assert torch.equal(q1.view(torch.int16), q2.view(torch.int16))
        d.duo_kv_append(one, kd, vd, slots, pos, 1e5, eps, kg, qd, qg, out=qd)  # queries in place, the cache written again
        assert torch.equal(qd.view(torch.int16), q2.view(torch.int16)) and torch.equal(one.data, two.data)
    else:
        assert q1 is None
    assert torch.equal(kd.cpu().view(torch.int16), K.view(torch.int16))


@pytest.mark.parametrize("fmt", ["bf16", "int8", "int4"])
def test_append_against_the_reference(duo_lib, fmt):
    """The stored keys as numbers, against float64: the rounding to bf16 (2^-8) with the fp32 errors
    above, and for codes half a step (s / 2) and the step's own rounding (2^-8 of it for each of up to 127)."""
    say("append against float64", fmt)
    d, m, kv, hd = duo_lib, 65, 2, 128
    K, V = rows(m, kv * hd, 3), rows(m, kv * hd, 4)
    pos = torch.arange(m, dtype=torch.int32) * 911
    cache = d.KVCache.empty(8, 16, kv, hd, fmt, DEV)
    slots = torch.arange(m, device=DEV)
    kg = gains(hd, 1, torch.bfloat16)
    assert d.duo_kv_append(cache, K.to(DEV), V.to(DEV), slots, pos.to(DEV), 1e4, 1e-6, kg.to(DEV)) is None
    k, _ = d.duo_kv_read(cache, slots)
    normed = S.head_norm(f64(K), kv, hd, f64(kg), 1e-6)
    ref = S.rope_at(normed, kv, hd, pos.numpy(), 1e4)
    size = np.abs(normed.reshape(m, kv, 2, -1)).sum(2, keepdims=True).repeat(2, 2).reshape(m, -1)
    tol = 2.0 ** -8 * 1.02 * np.abs(ref) + (2.0 ** -22 + (hd / 2 + 16) * 2.0 ** -24) * size
    if fmt != "bf16":
        top = np.abs(ref.reshape(m, -1, 32)).max(-1).repeat(32, -1) * (1 + 2.0 ** -7)
        step = top / S.MOST[fmt]
        # the number read back is rounded to bf16 once more
        tol = tol + step / 2 * (1 + 2.0 ** -7) + 2.0 ** -8 * np.abs(ref) + 2.0 ** -8 * (np.abs(ref) + step)
    assert (np.abs(f64(k) - ref) <= tol).all()


def test_other_stream_and_graph(duo_lib):
    """Work goes to the current stream; a captured append replays on new contents."""
    say("append on another stream and in a graph")
    d, m, kv, hd = duo_lib, 40, 2, 64
    K, V, Q = (rows(m, n * hd, 20 + i).to(DEV) for i, n in enumerate((kv, kv, 8)))
    pos, slots = torch.arange(m, device=DEV, dtype=torch.int32), torch.arange(m, device=DEV)
    ref, cache = (d.KVCache(torch.zeros_like(d.KVCache.empty(3, 16, kv, hd, "int8", DEV).data), 16, kv, hd, "int8") for _ in range(2))
    out = torch.empty_like(Q)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        d.duo_kv_append(cache, K, V, slots, pos, Q=Q, out=out)
    torch.cuda.current_stream().wait_stream(s)
    want = d.duo_kv_append(ref, K, V, slots, pos, Q=Q)
    assert torch.equal(out, want) and torch.equal(ref.data, cache.data)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        d.duo_kv_append(cache, K, V, slots, pos, Q=Q, out=out)
    for i in range(3):
        K.copy_(rows(m, kv * hd, 50 + i))
        Q.copy_(rows(m, 8 * hd, 60 + i))
        pos.add_(m)
        g.replay()
        want = d.duo_kv_append(ref, K, V, slots, pos, Q=Q)
        torch.cuda.synchronize()
        assert torch.equal(out, want) and torch.equal(ref.data, cache.data)

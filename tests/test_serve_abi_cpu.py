"""Host-side checks of the serving entry points (no GPU needed): argument errors
come back before any device work, valid arguments reach DUO_ERR_NO_DEVICE here;
sizes of pages and workspaces; and pins of the float64 reference."""

import ctypes

import numpy as np
import pytest
import torch

from oracle import serve_ref as S

FAKE = ctypes.c_void_p(1 << 20)      # never dereferenced on the host
WS = ctypes.c_void_p(256 << 20)
BIG = 10 ** 12


@pytest.fixture()
def codes(duo_lib):
    d = duo_lib
    if torch.cuda.device_count():
        pytest.skip("valid arguments with made-up addresses would be launched")
    return d.lib(), d.DUO_OK, d.DUO_ERR_INVALID_ARG, d.DUO_ERR_UNSUPPORTED, d.DUO_ERR_NO_DEVICE


def test_rope_at(codes):
    L, OK, E, UNS, NODEV = codes
    call = lambda X=FAKE, m=8, h=2, hd=64, ldx=128, pos=FAKE, th=1e4, Y=WS, ldy=128: L.duo_rope_at(X, m, h, hd, ldx, pos, th, Y,
                                                                                               ldy, None)
    assert call() == NODEV
    assert call(Y=FAKE) == NODEV                       # in place
    assert call(Y=FAKE, ldy=136) == E                  # in place with another stride
    assert call(m=0, X=None, Y=None, pos=None) == OK
    for bad in (dict(m=-1), dict(h=0), dict(hd=63), dict(hd=0), dict(ldx=127), dict(ldy=127), dict(th=0.0),
                dict(th=float("nan")), dict(th=float("inf")), dict(X=None), dict(Y=None), dict(pos=None)):
        assert call(**bad) == E, bad
    assert call(hd=258, ldx=1024, ldy=1024) == UNS
    assert call(m=1 << 31) == UNS


def _cache(data=FAKE.value, pages=10, page=16, kv=2, hd=64, fmt=0):
    from paper_2506_20194_amd.duo import KvCache

    return ctypes.byref(KvCache(data, pages, page, kv, hd, fmt))


BAD_CACHES = [dict(data=None), dict(data=FAKE.value + 8), dict(pages=0), dict(pages=-1), dict(page=0), dict(page=-16), dict(kv=0),
              dict(hd=0), dict(fmt=3), dict(fmt=-1)]
ODD_CACHES = [dict(page=8), dict(page=48), dict(page=512), dict(hd=96), dict(hd=256), dict(kv=65536), dict(pages=1 << 31)]


@pytest.mark.parametrize("entry", ["duo_kv_write", "duo_kv_read"])
def test_cache_rows(codes, entry):
    L, OK, E, UNS, NODEV = codes

    def call(cache=None, K=FAKE, ldk=128, V=FAKE, ldv=128, slots=FAKE, m=5):
        c = cache or _cache()
        if entry == "duo_kv_write":
            return L.duo_kv_write(c, K, ldk, V, ldv, slots, m, None)
        return L.duo_kv_read(c, slots, m, K, ldk, V, ldv, None)

    assert call() == NODEV
    assert all(call(_cache(fmt=f)) == NODEV for f in (0, 1, 2))
    assert call(m=0, K=None, V=None, slots=None) == OK
    assert all(call(_cache(**b)) == E for b in BAD_CACHES)
    assert all(call(_cache(**b), ldk=1 << 24, ldv=1 << 24) == UNS for b in ODD_CACHES)
    for bad in (dict(m=-1), dict(K=None), dict(V=None), dict(slots=None), dict(ldk=127), dict(ldv=120)):
        assert call(**bad) == E, bad
    for odd in (dict(ldk=132), dict(ldv=129), dict(K=ctypes.c_void_p(FAKE.value + 2)), dict(V=ctypes.c_void_p(FAKE.value + 8)),
                dict(m=1 << 31)):
        assert call(**odd) == UNS, odd


def test_page_bytes(duo_lib):
    b = duo_lib.lib().duo_kv_page_bytes
    for i, fmt in enumerate(("bf16", "int8", "int4")):
        for page in (16, 32, 64, 128, 256):
            for hd in (64, 128):
                assert b(i, page, 5, hd) == 5 * S.block_bytes(page, hd, fmt)
    assert b(0, 16, 0, 64) == b(0, 16, 2, 32) == b(3, 16, 2, 64) == b(0, 24, 2, 64) == b(0, -16, 2, 64) == 0


def test_attention_packed(codes):
    L, OK, E, UNS, NODEV = codes

    def call(Q=FAKE, ldq=256, K=FAKE, ldk=128, V=FAKE, ldv=128, cq=FAKE, tq=10, ck=FAKE, tk=20, n=2, h=4, kv=2, hd=64, sc=0.1,
             O=FAKE, ldo=256, ws=None, wsb=0):
        return L.duo_attention_packed(Q, ldq, K, ldk, V, ldv, cq, tq, ck, tk, n, h, kv, hd, sc, O, ldo, ws, wsb, None)

    assert call() == NODEV
    assert call(ck=None, tk=10) == NODEV
    assert call(tk=0, K=None, V=None) == NODEV          # no keys at all: rows of zeros
    assert call(ldo=257) == NODEV
    assert call(n=0) == OK and call(tq=0, Q=None, O=None) == OK
    for bad in (dict(Q=None), dict(K=None), dict(V=None), dict(cq=None), dict(O=None), dict(ck=None), dict(tq=-1), dict(tk=-1),
                dict(n=-1), dict(h=0), dict(kv=0), dict(kv=3), dict(kv=8), dict(hd=0), dict(sc=float("nan")),
                dict(sc=float("inf")), dict(ldq=255), dict(ldk=127), dict(ldv=127), dict(ldo=255)):
        assert call(**bad) == E, bad
    for odd in (dict(hd=32), dict(ldq=260), dict(ldk=132), dict(ldv=130), dict(Q=ctypes.c_void_p(FAKE.value + 2)),
                dict(K=ctypes.c_void_p(FAKE.value + 8)), dict(V=ctypes.c_void_p(FAKE.value + 4)), dict(ldk=1 << 24), dict(tq=1 << 31),
                dict(tk=1 << 31)):
        assert call(**odd) == UNS, odd


def test_attention_packed_workspace(codes, duo_lib):
    """Nothing but few queries on long sequences is split and needs scratch memory."""
    L, OK, E, UNS, NODEV = codes
    size = L.duo_attention_packed_workspace_size
    assert size(10, 20, 2, 4, 2, 64) == size(100000, 100000, 10, 32, 32, 128) == size(10, 100000, 0, 4, 2, 64) == 0
    assert size(1, 100000, 1, 4, 3, 64) == size(1, 100000, 1, 4, 2, 32) == size(0, 100000, 1, 4, 2, 64) == 0
    need = size(1, 100000, 1, 4, 2, 64)
    assert 0 < need < 1 << 26
    call = lambda ws, wsb: L.duo_attention_packed(FAKE, 256, FAKE, 128, FAKE, 128, FAKE, 1, FAKE, 100000, 1, 4, 2, 64, 0.1, FAKE,
                                                  256, ws, wsb, None)
    assert call(WS, need) == NODEV
    for ws, wsb in ((None, 0), (WS, need - 1), (ctypes.c_void_p(WS.value + 64), BIG)):
        assert call(ws, wsb) == duo_lib.DUO_ERR_WORKSPACE


def test_attention_paged(codes, duo_lib):
    L, OK, E, UNS, NODEV = codes

    def call(Q=FAKE, ldq=256, cache=None, table=FAKE, ldt=8, lens=FAKE, n=3, most=128, h=4, sc=0.1, O=FAKE, ldo=256, ws=WS,
             wsb=BIG):
        return L.duo_attention_paged(Q, ldq, cache or _cache(), table, ldt, lens, n, most, h, sc, O, ldo, ws, wsb, None)

    assert call() == NODEV
    assert call(ldt=9, most=129) == NODEV
    assert call(most=0, table=None, ldt=0) == NODEV      # nothing cached: rows of zeros
    assert call(n=0, Q=None) == OK
    assert all(call(cache=_cache(**b)) == E for b in BAD_CACHES)
    for bad in (dict(Q=None), dict(table=None), dict(lens=None), dict(O=None), dict(n=-1), dict(most=-1), dict(h=0), dict(h=3),
                dict(ldt=7), dict(ldt=-1), dict(ldq=255), dict(ldo=255), dict(sc=float("nan"))):
        assert call(**bad) == E, bad
    for odd in (dict(ldq=260), dict(Q=ctypes.c_void_p(FAKE.value + 8)), dict(n=1 << 31)):
        assert call(**odd) == UNS, odd
    size = L.duo_attention_paged_workspace_size
    if size(3, 4, 2, 64, 100000):
        long = dict(ldt=10000, most=100000)
        assert call(**long, wsb=size(3, 4, 2, 64, 100000)) == NODEV
        for ws in (dict(ws=None), dict(wsb=16), dict(ws=ctypes.c_void_p(WS.value + 8))):
            assert call(**long, **ws) == duo_lib.DUO_ERR_WORKSPACE, ws
    assert size(-1, 4, 2, 64, 100) == size(3, 0, 2, 64, 100) == size(3, 4, 2, 64, 0) == 0


@pytest.mark.parametrize("heads,kv,hd", [(1, 1, 64), (64, 8, 128), (32, 32, 128), (24, 1, 64)])
def test_paged_workspace_never_falls(duo_lib, heads, kv, hd):
    size = duo_lib.lib().duo_attention_paged_workspace_size
    lengths = sorted({int(1.1 ** i) for i in range(140)})
    for n in (1, 2, 7, 48, 300):
        s = [size(n, heads, kv, hd, x) for x in lengths]
        assert s == sorted(s)
    for x in (1, 100, 3000, 100000):
        s = [size(n, heads, kv, hd, x) for n in range(1, 400)]
        assert s == sorted(s)


def test_binding_refuses_host_tensors(duo_lib):
    d = duo_lib
    if torch.cuda.device_count():
        pytest.skip("valid arguments with made-up addresses would be launched")
    cache = d.KVCache(torch.zeros((2, 1, d.kv_page_bytes(16, 1, 64)), dtype=torch.uint8), 16, 1, 64)
    x = torch.zeros((3, 64), dtype=torch.bfloat16)
    i = torch.zeros(3, dtype=torch.int64)
    with pytest.raises(ValueError):
        d.duo_kv_write(cache, x, x, i)
    with pytest.raises(ValueError):
        d.duo_kv_read(cache, i)
    with pytest.raises(ValueError):
        d.duo_rope_at(x, 1, 64, i.int())
    with pytest.raises(ValueError):
        d.duo_attention_packed(x, x, x, torch.tensor([0, 3], dtype=torch.int32), 1, 1, 64)
    with pytest.raises(ValueError):
        d.duo_attention_paged(x, cache, torch.zeros((3, 1), dtype=torch.int32), i.int(), 1)


def test_cache_object(duo_lib):
    d = duo_lib
    if torch.cuda.device_count():
        pytest.skip("valid arguments with made-up addresses would be launched")
    cache = d.KVCache(torch.zeros((5, 2, d.kv_page_bytes(32, 2, 64, "int4") // 2), dtype=torch.uint8), 32, 2, 64, "int4")
    table = torch.tensor([[3, 1], [0, 4]], dtype=torch.int32)
    s = cache.slots(table, torch.tensor([0, 0, 1]), torch.tensor([31, 32, 63]))
    assert s.tolist() == [3 * 32 + 31, 32, 4 * 32 + 31] and s.dtype == torch.int64


# the reference ------------------------------------------------------------

def test_reference_quantisation_by_hand():
    x = np.zeros((1, 1, 64))
    x[0, 0, 0], x[0, 0, 1], x[0, 0, 2], x[0, 0, 3] = 127.0, 0.5, 1.5, -2.5
    x[0, 0, 40] = -14.0
    c, s = S.quantize(x, "int8")
    assert s[0, 0].tolist() == [1.0, float(S.bf16(14 / 127))]
    assert c[0, 0, :4].tolist() == [127, 0, 2, -2] and c[0, 0, 40] == -127
    c, s = S.quantize(x, "int4")
    assert s[0, 0].tolist() == [float(S.bf16(127 / 7)), 2.0] and c[0, 0, 40] == -7
    data = np.full((2, 1, S.block_bytes(16, 64, "int4")), 9, dtype=np.uint8)
    out = S.write(data, x, x, np.array([16 + 3]), 16, 64, "int4")
    assert (out[0] == 9).all() and out[1, 0, 3 * 32 + 20] == 1 | 8 << 4  # channel 40: -7 + 8; channel 41: 0 + 8
    assert out[1, 0, 2 * 16 * 32 + 3 * 4 + 2:2 * 16 * 32 + 3 * 4 + 4].tolist() == [0x00, 0x40]  # 2.0


def test_reference_attention_is_softmax():
    g = torch.Generator().manual_seed(0)
    q, k, v = (torch.randn(s, generator=g, dtype=torch.float64) for s in ((5, 4, 8), (9, 2, 8), (9, 2, 8)))
    O, tol = S.attend(q.numpy(), k.numpy(), v.numpy(), 0.3, S.causal(5, 9))
    m = torch.ones((5, 9), dtype=torch.bool).tril(4)
    ref = torch.nn.functional.scaled_dot_product_attention(q.transpose(0, 1), k.repeat_interleave(2, 1).transpose(0, 1),
                                                           v.repeat_interleave(2, 1).transpose(0, 1), m, scale=0.3)
    assert np.allclose(O, ref.transpose(0, 1).numpy(), rtol=1e-12)
    O, _ = S.attend(q.numpy(), k.numpy()[:3], v.numpy()[:3], 0.3, S.causal(5, 3))
    assert (O[:2] == 0).all() and (O[2:] != 0).all()


def test_reference_rotation():
    x = np.arange(16.0).reshape(2, 8)
    y = S.rope_at(x, 1, 8, np.array([0, 3]), 100.0)
    assert np.allclose(y[0], x[0])
    for i in range(4):
        a = 3 * 100.0 ** (-i / 4)
        z = (x[1, i] + 1j * x[1, i + 4]) * np.exp(1j * a)
        assert np.allclose((y[1, i], y[1, i + 4]), (z.real, z.imag))

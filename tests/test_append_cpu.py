"""Host-side checks of the head norms with rotation and of the append to the cache (no GPU
needed): argument errors come back before any device work, valid arguments reach
DUO_ERR_NO_DEVICE here; the binding's own refusals; a pin of the reference."""

import ctypes

import numpy as np
import pytest
import torch

from oracle import serve_ref as S

FAKE = ctypes.c_void_p(1 << 20)  # never dereferenced on the host
OUT = ctypes.c_void_p(256 << 20)


@pytest.fixture()
def codes(duo_lib):
    d = duo_lib
    if torch.cuda.device_count():
        pytest.skip("valid arguments with made-up addresses would be launched")
    return d.lib(), d.DUO_OK, d.DUO_ERR_INVALID_ARG, d.DUO_ERR_UNSUPPORTED, d.DUO_ERR_NO_DEVICE


def test_head_norm_rope(codes):
    L, OK, E, UNS, NODEV = codes

    def call(X=FAKE, m=8, h=2, hd=64, ldx=128, pos=FAKE, gain=FAKE, dt=1, eps=1e-5, th=1e4, Y=OUT, ldy=128):
        return L.duo_head_norm_rope(X, m, h, hd, ldx, pos, gain, dt, eps, th, Y, ldy, None)

    assert call() == call(dt=0) == call(gain=None, dt=7) == call(eps=0.0) == call(Y=FAKE) == NODEV
    assert call(ldx=129, ldy=133) == call(hd=62) == NODEV  # rows of any alignment
    assert call(m=0, X=None, Y=None, pos=None) == OK
    for bad in (dict(m=-1), dict(h=0), dict(hd=63), dict(hd=0), dict(ldx=127), dict(ldy=127), dict(th=0.0), dict(dt=2), dict(dt=-1),
                dict(th=float("nan")), dict(th=float("inf")), dict(X=None), dict(Y=None), dict(pos=None), dict(eps=-1e-9),
                dict(eps=float("nan")), dict(eps=float("inf")), dict(Y=FAKE, ldy=136)):
        assert call(**bad) == E, bad
    assert call(hd=258, ldx=1024, ldy=1024) == call(m=1 << 31) == UNS


def _cache(data=FAKE.value, pages=10, page=16, kv=2, hd=64, fmt=0):
    from paper_2506_20194_amd.duo import KvCache

    return ctypes.byref(KvCache(data, pages, page, kv, hd, fmt))


def test_kv_append(codes):
    L, OK, E, UNS, NODEV = codes

    def call(cache=None, K=FAKE, ldk=128, V=FAKE, ldv=128, slots=FAKE, pos=FAKE, m=5, th=1e4, eps=1e-5, kg=FAKE, Q=FAKE, ldq=256,
             h=4, qg=FAKE, dt=1, Y=OUT, ldy=256):
        return L.duo_kv_append(cache or _cache(), K, ldk, V, ldv, slots, pos, m, th, eps, kg, Q, ldq, h, qg, dt, Y, ldy, None)

    for good in (dict(), dict(dt=0), dict(eps=-1.0, kg=None, qg=None, dt=9), dict(kg=None, qg=None), dict(Y=FAKE),
                 dict(h=0, Q=None, Y=None, qg=None, ldq=0, ldy=0), dict(h=5, ldq=320, ldy=328), dict(eps=0.0)):
        assert call(**good) == NODEV, good
    assert call(m=0, K=None, V=None, Q=None, Y=None, slots=None, pos=None) == OK
    for bad in (dict(m=-1), dict(ldk=127), dict(ldv=127), dict(ldq=255), dict(ldy=255), dict(th=0.0), dict(th=float("nan")),
                dict(eps=float("nan")), dict(eps=float("inf")), dict(eps=-1.0), dict(dt=2), dict(h=-1), dict(h=65536),
                dict(K=None), dict(V=None), dict(Q=None), dict(Y=None), dict(slots=None), dict(pos=None), dict(Y=FAKE, ldy=264),
                dict(h=0, ldq=0, ldy=0), dict(cache=_cache(data=None)), dict(cache=_cache(pages=0)), dict(cache=_cache(fmt=3))):
        assert call(**bad) == E, bad
    for odd in (dict(ldk=132), dict(ldv=132), dict(ldq=260), dict(ldy=260), dict(K=ctypes.c_void_p(FAKE.value + 8)),
                dict(V=ctypes.c_void_p(FAKE.value + 8)), dict(Q=ctypes.c_void_p(FAKE.value + 8)),
                dict(Y=ctypes.c_void_p(OUT.value + 8)), dict(m=1 << 31), dict(cache=_cache(page=8)), dict(cache=_cache(hd=96))):
        assert call(**odd) == UNS, odd


def test_binding(duo_lib):
    d = duo_lib
    b = lambda *s: torch.zeros(s, dtype=torch.bfloat16)
    pos, slots = torch.zeros(3, dtype=torch.int32), torch.zeros(3, dtype=torch.int64)
    cache = d.KVCache.empty(2, 16, 2, 64, "int8", "cpu")
    with pytest.raises(ValueError, match="HIP"):
        d.duo_head_norm_rope(b(3, 128), 2, 64, pos)
    with pytest.raises(ValueError, match="HIP"):
        d.duo_kv_append(cache, b(3, 128), b(3, 128), slots, pos)
    with pytest.raises(ValueError, match="multiple"):
        d.duo_kv_append(cache, b(3, 128), b(3, 128), slots, pos, Q=b(3, 100))
    with pytest.raises(ValueError, match="belong to Q"):
        d.duo_kv_append(cache, b(3, 128), b(3, 128), slots, pos, eps=1e-5, q_gain=b(64))
    with pytest.raises(ValueError, match="belong to a norm"):
        d.duo_kv_append(cache, b(3, 128), b(3, 128), slots, pos, k_gain=b(64))
    with pytest.raises(ValueError, match="negative"):
        d.duo_kv_append(cache, b(3, 128), b(3, 128), slots, pos, eps=-1.0)


def test_head_norm_pin():
    """A head of one number is its sign; a scale leaves a head as it is; hand-worked values."""
    x = np.array([[3.0, 4.0, -2.0, 0.0]])
    assert np.allclose(S.head_norm(x[:, :3], 3, 1, eps=0.0), [[1, 1, -1]])
    y = S.head_norm(x, 2, 2, [2.0, 1.0], 0.0)
    assert np.allclose(y, [[3 / 12.5 ** 0.5 * 2, 4 / 12.5 ** 0.5, -(2.0 ** 0.5) * 2, 0.0]])
    assert np.allclose(S.head_norm(5 * x, 2, 2, eps=0.0), S.head_norm(x, 2, 2, eps=0.0))

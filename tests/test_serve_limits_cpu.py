"""Launches of the serving operators stay below 2^32 work items in an axis: what would need
more is refused before anything is enqueued (no GPU needed)."""

import ctypes

import pytest
import torch

FAKE = ctypes.c_void_p(1 << 20)  # never dereferenced on the host


@pytest.fixture()
def lib(duo_lib):
    if torch.cuda.device_count():
        pytest.skip("valid arguments with made-up addresses would be launched")
    return duo_lib


@pytest.mark.parametrize("kv", [1, 3, 8, 12])
def test_packed_blocks(lib, kv):
    """One-token sequences: about two blocks of rows each, for every K/V head, and 256
    threads for each."""
    call = lambda n: lib.lib().duo_attention_packed(FAKE, kv * 64, FAKE, kv * 64, FAKE, kv * 64, FAKE, n, FAKE, n, n, kv, kv, 64,
                                                    0.1, FAKE, kv * 64, None, 0, None)
    most = (2 ** 32 // 256) // kv  # blocks of a K/V head, n (1 + 1 / 128) of n sequences
    assert call(int(most * 0.98)) == lib.DUO_ERR_NO_DEVICE
    assert call(int(most * 1.01)) == lib.DUO_ERR_UNSUPPORTED


def test_cache_rows(lib):
    from paper_2506_20194_amd.duo import KvCache

    c = ctypes.byref(KvCache(FAKE.value, 10, 16, 1, 128, 0))
    for entry in ("duo_kv_write", "duo_kv_read"):
        for m, want in (((1 << 30) - 1, lib.DUO_ERR_NO_DEVICE), (1 << 30, lib.DUO_ERR_UNSUPPORTED)):
            args = (c, FAKE, 128, FAKE, 128, FAKE, m, None) if entry == "duo_kv_write" else (c, FAKE, m, FAKE, 128, FAKE, 128, None)
            assert getattr(lib.lib(), entry)(*args) == want


def test_rotated_rows(lib):
    """More rows per workgroup instead, as long as their angles fit it (64 KiB: 64 rows of 128
    pairs, 2^30 rows)."""
    call = lambda m, h, hd: lib.lib().duo_rope_at(FAKE, m, h, hd, h * hd, FAKE, 1e4, FAKE, h * hd, None)
    assert call(2 ** 24 + 5, 129, 2) == call(2 ** 31 - 1, 4, 64) == call(2 ** 30 - 64, 33, 256) == lib.DUO_ERR_NO_DEVICE
    assert call(2 ** 31 - 1, 33, 256) == lib.DUO_ERR_UNSUPPORTED

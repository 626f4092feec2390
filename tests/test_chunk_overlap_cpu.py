"""An output of the attention of chunks that has bytes of the queries' matrix: one workgroup would
write what another still has to read.  Refused on the host; matrices beside each other, as
columns of one wider matrix too, are not (no GPU needed: they reach DUO_ERR_NO_DEVICE here)."""

import ctypes

import pytest
import torch

BASE = 1 << 20  # never dereferenced on the host
W = 256         # numbers of a row: 4 heads of 64


@pytest.fixture()
def call(duo_lib):
    d = duo_lib
    if torch.cuda.device_count():
        pytest.skip("valid arguments with made-up addresses would be launched")
    P = ctypes.c_void_p
    cache = ctypes.byref(d.KvCache(1 << 30, 10, 16, 2, 64, 0))

    def f(q, ldq, o, ldo, rows=8):
        return d.lib().duo_attention_chunk(P(BASE + 2 * q), ldq, rows, cache, P(2 << 30), 4, P(2 << 30), P(2 << 30), 3, rows, 64, 4, 0, 0,
                                           0.125, P(BASE + 2 * o), ldo, P(4 << 30), 1 << 40, None)

    return f, d.DUO_ERR_INVALID_ARG, d.DUO_ERR_NO_DEVICE


def test_shifted(call):
    """Slices of one matrix: rows 0 .. 7 and rows k .. k + 7, or k numbers further on."""
    f, bad, good = call
    for k in range(-7, 8):
        assert f(8 * W, W, (8 + k) * W, W) == bad, k
    assert f(8 * W, W, 16 * W, W) == f(8 * W, W, 0, W) == good
    for k in (-8 * W + 8, -W, -8, -1, 1, 8, W - 8, 7 * W + 8, 8 * W - 8):
        assert f(8 * W, W, 8 * W + k, W) == bad, k
        if k % 8 == 0:
            assert f(8 * W + k, W, 8 * W, W) == bad, k


def test_beside_each_other(call):
    """Columns of a wider matrix: apart, touching, one number in common, around the ends."""
    f, bad, good = call
    for ld in (2 * W, 3 * W, 3 * W + 8):
        for k in range(-3, 4):
            for col in (W, ld - W):
                assert f(4 * ld, ld, 4 * ld + k * ld + col, ld) == good, (ld, k, col)
            for col in (0, 1, W - 1, ld - W + 1, ld - 1):
                assert f(4 * ld, ld, 4 * ld + k * ld + col, ld) == bad, (ld, k, col)
    # the first number behind the last row, and the last before the first
    ld = 3 * W
    assert f(0, ld, 7 * ld + W, ld) == f(7 * ld + W, ld, 0, ld) == good
    assert f(0, ld, 7 * ld + W - 1, ld) == bad


def test_strides_of_two_lengths(call):
    f, bad, good = call
    assert f(0, W, 8 * W, 2 * W) == f(15 * W, W, 0, 2 * W) == good
    assert f(0, W, 8 * W - 1, 2 * W) == f(14 * W, W, 0, 2 * W) == bad
    assert f(0, W, 4 * W, 2 * W) == bad


def test_one_row(call):
    """A single row has no stride to speak of."""
    f, bad, good = call
    assert f(W, 99 * W, 0, W, 1) == f(W, W, 2 * W, 99 * W, 1) == f(0, 4 * W, 2 * W, 4 * W, 1) == good
    for k in (-W + 1, -1, 0, 1, W - 1):
        assert f(W, 2 * W, W + k, 2 * W, 1) == bad

"""Pins of the serving reference's bounds: a comparison with them accepts what is
right and refuses one wrong element, wherever it stands."""

import numpy as np
import pytest

from oracle import serve_ref as S

import test_packed_gpu


@pytest.mark.parametrize("lq,lk", [(5, 0), (5, 3), (4, 9)])
def test_bound_is_positive(lq, lk):
    """Also where no key is seen and the output is an exact 0: a quotient of error
    and bound is then a number."""
    g = np.random.default_rng(0)
    Q, K, V = g.standard_normal((lq, 4, 8)), g.standard_normal((lk, 2, 8)), g.standard_normal((lk, 2, 8))
    _, bound = S.attend(Q, K, V, 0.3, S.causal(lq, lk))
    assert (bound > 0).all()


@pytest.mark.parametrize("lq,lk", [([5], [0]), ([3, 5, 2], [3, 0, 7]), ([70, 1], [0, 0])])
def test_one_wrong_element_without_keys(lq, lk):
    g = np.random.default_rng(1)
    heads, kv, hd = 2, 1, 64
    Q, K, V = g.standard_normal((sum(lq), heads * hd)), g.standard_normal((sum(lk), kv * hd)), g.standard_normal((sum(lk), kv * hd))
    O, a, b = [], 0, 0
    for n, m in zip(lq, lk):
        O.append(S.attend(Q[a:a + n].reshape(n, heads, hd), K[b:b + m].reshape(m, kv, hd), V[b:b + m].reshape(m, kv, hd),
                          hd ** -0.5, S.causal(n, m))[0].reshape(n, -1))
        a, b = a + n, b + m
    O = np.concatenate(O)
    test_packed_gpu.check(O, Q, K, V, lq, lk, heads, kv, hd)
    row = int(np.cumsum([0] + lq)[lk.index(0)])  # first of a sequence without keys
    for at in ((row, 0), (row, heads * hd - 1), (row + lq[lk.index(0)] - 1, 7)):
        wrong = O.copy()
        wrong[at] += 1e-6
        with pytest.raises(AssertionError):
            test_packed_gpu.check(wrong, Q, K, V, lq, lk, heads, kv, hd)

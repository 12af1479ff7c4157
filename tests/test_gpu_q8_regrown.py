"""Integers of the 8-bit block cache whose block's scale grows: older codes c become the nearest to c before / now, ties to the even
one, by integer arithmetic here."""
from fractions import Fraction

import numpy as np
import pytest
import torch

import paper_2405_03917_amd as cq
from q8_util import D, TILE, Cache

pytestmark = pytest.mark.gpu

CODES = np.arange(-127, 128)
ROWS = 2                                                     # tokens that hold every code once


def _grown(first, second, n_old, m):
    """Older codes of keys and of (negative) values after a block of n_old tokens, largest magnitude `first`, took m tokens of `second`."""
    before, now = np.float32(first / 127.0), np.float32(second / 127.0)
    x = np.zeros((TILE, D))
    flat = x[n_old - ROWS:n_old].reshape(-1)
    flat[:CODES.size] = (CODES * np.float64(before)).astype(np.float16)
    flat[-1] = first
    x[n_old:n_old + m, 3] = second
    assert np.array_equal(x, x.astype(np.float16))
    assert np.array_equal(np.rint(flat[:CODES.size] / before), CODES)        # (a code is 2^-11 of itself off at most)
    x = torch.from_numpy(x).half().cuda().view(1, TILE, D)
    cache = Cache("int8", 1, 1, TILE, seed=1)
    cq.cq_append_q8(x[:, :n_old], -x[:, :n_old], cache.dev, cache.fmt, n_old, TILE)
    cq.cq_append_q8(x[:, n_old:n_old + m], -x[:, n_old:n_old + m], cache.dev, cache.fmt, n_old + m, TILE)
    k, v, ks, vs = cache.download()
    assert ks.item() == vs.item() == now
    want = np.array([round(Fraction(int(c)) * Fraction(float(before)) / Fraction(float(now))) for c in CODES])    # (half to even)
    old = lambda a: a[n_old - ROWS:n_old].reshape(-1)[:CODES.size].astype(np.int64) - 128  # noqa: E731
    return old(k[0, 0, 0]), -old(v[0, 0, 0].T), want


@pytest.mark.parametrize("n_old,m", [(2, 1), (2, 5), (18, 1), (18, 2), (35, 1), (35, 29)])
@pytest.mark.parametrize("largest", [1.0, 1.021484375, 1.0244140625, 700.5])
def test_a_scale_that_doubles(largest, n_old, m):
    """Every odd code is a tie, whatever the reciprocal of the scale rounds to."""
    k, v, want = _grown(largest, 2 * largest, n_old, m)
    assert np.array_equal(want, np.rint(CODES / 2))
    assert np.array_equal(k, want) and np.array_equal(v, want)


@pytest.mark.parametrize("n_old,m", [(2, 1), (2, 5), (18, 1), (35, 29)])
@pytest.mark.parametrize("before,now", [(3, 10), (1, 6), (5, 14), (7, 10), (11, 14), (1, 14), (9, 16), (13, 15)])
@pytest.mark.parametrize("unit", [1.0, 2.0 ** -9])
def test_ties_under_ratios_that_are_no_numbers(before, now, unit, n_old, m):
    """Scales of small integers: c before / now is a tie for some codes though before / now itself is rounded."""
    k, v, want = _grown(127 * before * unit, 127 * now * unit, n_old, m)
    assert np.array_equal(k, want) and np.array_equal(v, want)

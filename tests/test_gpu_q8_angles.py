"""The angles of cq_append_q8 against decimals of 60 digits: a cosine or sine is off by 2^-50 + 2^-51 p theta at most, the rounding of a frequency
(2^-52 of it, a power function's last place), of its product with a position (2^-53) and of a handful of operations on the results."""
from decimal import Decimal, localcontext

import numpy as np
import pytest

import paper_2405_03917_amd as cq

pytestmark = pytest.mark.gpu
PI = Decimal("3.14159265358979323846264338327950288419716939937510582097494459230781640628621")


def _exact(base, i, p):
    """cos, sin of p base^(-2 i / 128), and that angle"""
    with localcontext() as c:
        c.prec = 60
        angle = p * (Decimal(base).ln() * -i / 64).exp()
        x = angle % (2 * PI)
        x = x - 2 * PI if x > PI else x
        total, term, n = [Decimal(0), Decimal(0)], Decimal(1), 0
        while abs(term) > Decimal(10) ** -50:
            total[n % 2] += term if n % 4 < 2 else -term
            n += 1
            term = term * x / n
        return total[0], total[1], float(angle)


@pytest.mark.parametrize("base", [10000, 500000])
def test_angles_to_the_last_position(base):
    positions = 1 << 20
    table = cq.Q8RopeTable(float(base), positions).table.cpu().numpy().view(np.float64).reshape(-1, 2)
    tiles = table[:positions // 64 * 64].reshape(-1, 64, 2)                  # [tile][pair]
    tokens = table[positions // 64 * 64:].reshape(16, 64, 4, 2)              # [pair % 16][token][pair / 16]
    worst = 0.0
    for p in (0, 1, 63, 64, 300, 4095, 6000, 32767, 131071, positions - 1):
        tile, u = divmod(p, 64)
        for i in range(64):
            a, b = tiles[tile, i], tokens[i % 16, u, i // 16]
            for got, at in ((a, 64 * tile), (b, u), ((a[0] * b[0] - a[1] * b[1], a[1] * b[0] + a[0] * b[1]), p)):
                c, s, angle = _exact(base, i, at)
                off = max(abs(Decimal(float(got[0])) - c), abs(Decimal(float(got[1])) - s))
                bound = 2.0 ** -50 + 2.0 ** -51 * angle
                assert off <= Decimal(bound), (p, at, i, float(off), bound)
                worst = max(worst, float(off))
    assert worst < 2.0 ** -32

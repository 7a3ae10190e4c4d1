"""Float32 products by three bfloat16 pieces a factor (csrc/matrix_tile.hpp): what the six products that are made leave out, computed
exactly on the host.  The pieces are cut here as the kernels cut them: each is what the ones before leave, rounded to nearest even."""
from fractions import Fraction

import numpy as np
import pytest


def rounded(x):
    """float32 -> bfloat16 (nearest, ties to even), as a float32."""
    bits = x.view(np.uint32)
    return ((bits + np.uint32(0x7FFF) + ((bits >> np.uint32(16)) & np.uint32(1))) & np.uint32(0xFFFF0000)).view(np.float32)


def pieces(x):
    found = []
    for _ in range(3):
        found.append(rounded(x))
        x = x - found[-1]
    return found, x


def factors(seed):
    rng = np.random.default_rng(seed)
    x = (1 + rng.integers(0, 2 ** 23, 20_000) * 2.0 ** -23).astype(np.float32)
    x[:10_000] = (1 + 2.0 ** -8 - rng.integers(0, 2 ** 8, 10_000) * 2.0 ** -23).astype(np.float32)         # (large second pieces)
    x[0] = 1 + 2.0 ** -8 - 2.0 ** -16 + 2.0 ** -17 - 2.0 ** -23
    return x * np.where(rng.integers(0, 2, x.size) > 0, 1, -1).astype(np.float32)


@pytest.mark.parametrize("power", [-100, -40, 0, 100])
def test_three_pieces_are_the_whole(power):
    x = np.ldexp(factors(1), power)
    p, left = pieces(x)
    assert not left.any()
    size = 2.0 ** power
    assert np.abs(p[1]).max() <= size * 2.0 ** -8 and np.abs(p[2]).max() <= size * 2.0 ** -17


def test_what_six_products_leave_out():
    x, y = factors(2), factors(2)[::-1].copy()
    y[0] = x[0]
    (p, _), (q, _) = pieces(x), pieces(y)
    p, q = [v.astype(np.float64) for v in p], [v.astype(np.float64) for v in q]
    left = p[1] * q[2] + p[2] * q[1] + p[2] * q[2]              # (exact in 64 bits)
    share = np.abs(left) / np.abs(x.astype(np.float64) * y)
    assert share.max() < 2.0 ** -24
    assert share[0] > 1.9 * 2.0 ** -25                         # more than half a unit can be missing
    made = sum(Fraction(float(p[i][0])) * Fraction(float(q[j][0])) for i, j in ((2, 0), (0, 2), (1, 1), (1, 0), (0, 1), (0, 0)))
    assert abs(made - Fraction(float(x[0])) * Fraction(float(y[0]))) < Fraction(float(x[0])) * Fraction(float(y[0])) / 2 ** 24


def test_factors_without_pieces():
    assert np.isfinite(rounded(np.array([3.396e38, -3.396e38], np.float32))).all()
    assert np.isinf(rounded(np.array([3.3962e38, np.inf], np.float32))).all()

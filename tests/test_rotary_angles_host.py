"""The turns per position that a Rotary's handle holds, against 1 / (2 pi) to 400 bits: however many whole turns a position makes, the fraction
that is left is right to half a unit of 2^-64, and so the angle to 2^31 half units (3.7e-10 radian) at the farthest position."""
import ctypes
from fractions import Fraction

import numpy as np
import pytest


def arctan_of_inverse(x: int, one: int) -> int:
    total, power, k, sign = 0, one // x, 1, 1
    while power:
        total += sign * (power // k)
        power, k, sign = power // (x * x), k + 2, -sign
    return total


ONE = 1 << 400
TWO_PI = Fraction(8 * (4 * arctan_of_inverse(5, ONE) - arctan_of_inverse(239, ONE)), ONE)      # Machin


def steps_of(rotary) -> list[int]:
    """The handle begins with the pairs' turns per position in units of 2^-64."""
    return list(ctypes.cast(rotary.handle, ctypes.POINTER(ctypes.c_uint64))[: rotary.dim // 2])


def test_two_pi():
    assert abs(float(TWO_PI) - 2 * np.pi) == 0.0
    assert abs(TWO_PI - Fraction(31415926535897932384626433832795028841971693993751, 5 * 10 ** 48)) < Fraction(1, 10 ** 47)


def frequencies():
    g = np.random.default_rng(0)
    some = [0.0, 1.0, 100.1, 1000.3, 1235.0, 65535.7, 65536.0, -1.0, -65536.0, 2 * np.pi, np.nextafter(2 * np.pi, 0), 65535.999999999, 1e-4, 1e-18, 5e-20, 1e-300, 5e-324, -1e-19]
    drawn = np.concatenate([g.uniform(-65536, 65536, 40), 2.0 ** g.uniform(-70, 16, 60) * g.choice([-1, 1], 60)])
    whole = np.round(g.uniform(1, 10000, 10)) * 2 * np.pi                # next to whole turns
    return np.concatenate([some, drawn, whole])[:128]


def test_steps(bq):
    f = frequencies()
    assert len(f) == 128
    got = steps_of(bq.Rotary(256, frequencies=f))
    for x, step in zip(f, got):
        turns = Fraction(float(x)) / TWO_PI
        off = (Fraction(step, 1 << 64) - turns) % 1
        assert min(off, 1 - off) <= Fraction(1, 1 << 65) * (1 + Fraction(1, 10 ** 9)), x


@pytest.mark.parametrize("position", [2 ** 31 - 1, -2 ** 31, 123456789, 1])
def test_far_positions(bq, position):
    """The promised 10^-9 radian, by the 64-bit product that the kernels form."""
    f = frequencies()
    for x, step in zip(f, steps_of(bq.Rotary(256, frequencies=f))):
        angle = Fraction((step * position) % (1 << 64), 1 << 64) * TWO_PI
        off = (angle - Fraction(float(x)) * position) % TWO_PI
        assert float(min(off, TWO_PI - off)) <= 1e-9, x

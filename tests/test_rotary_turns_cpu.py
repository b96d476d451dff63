"""Frequencies as fractions of a turn against exact rational arithmetic.  No kernel runs.

A frequency is a double f; its fraction f / 2 pi in 2^-64 is cut from a product in two doubles (2^-105 of it), so that it is
off by less than one of them and positions up to 2^31 turn by f to 2^-33 of a turn.
"""
import ctypes
import random
from fractions import Fraction

import pytest

PI = Fraction(31415926535897932384626433832795028841971693993751058209749445923, 10 ** 64)


@pytest.fixture(scope="module")
def lib():
    from paper_2605_09681_gb300 import build, _lib
    build.build()
    return _lib.load()


def _turns(lib, freq):
    from paper_2605_09681_gb300._lib import FkRotary, FkRotaryConfig
    n = len(freq)
    c = FkRotaryConfig(2 * n, 2 * n, 0, 1, (ctypes.c_int32 * 4)(n), 0, 0, 1e4, 1.0, 1.0, 32.0, 0.0, (ctypes.c_double * n)(*freq))
    r = FkRotary()
    assert lib.fk_rotary_make(ctypes.byref(c), ctypes.byref(r)) == 0
    return list(r.turns)[:n]


@pytest.mark.parametrize("low,high", [(1.0, 3.1415926), (1e-3, 1.0), (1e-9, 1e-6), (1e-25, 1e-18), (1e-300, 1e-290)])
def test_given_frequencies_are_exact(lib, low, high):
    r = random.Random(int(1 / low) % 1000)
    freq = [r.choice([-1, 1]) * r.uniform(low, high) for _ in range(127)] + [high]
    for f, t in zip(freq, _turns(lib, freq)):
        got = t if f > 0 or t == 0 else t - (1 << 64)        # the two's complement of what turns backwards
        assert abs(got - Fraction(f) / (2 * PI) * (1 << 64)) <= 1, f


def test_edges(lib):
    half = 3.141592653589793                                 # below pi, but refused: the limit is 3.14159265358979
    freq = [0.0, -0.0, 3.1415926535897, -3.1415926535897, 5e-324, 1.0, 0.5, 0.25]
    t = _turns(lib, freq)
    assert t[0] == t[1] == 0 and t[2] + t[3] == 1 << 64 and t[4] == 0
    assert abs(t[5] - (1 << 64) / (2 * PI)) <= 1 and abs(t[5] - 2 * t[6]) <= 1 and abs(t[6] - 2 * t[7]) <= 1
    from paper_2605_09681_gb300._lib import FkRotary, FkRotaryConfig
    c = FkRotaryConfig(16, 16, 0, 1, (ctypes.c_int32 * 4)(8), 0, 0, 1e4, 1.0, 1.0, 32.0, 0.0, (ctypes.c_double * 8)(*[half] * 8))
    assert lib.fk_rotary_make(ctypes.byref(c), ctypes.byref(FkRotary())) == 1

"""The fractions of a circle that rotations are kept as, against integer arithmetic (CPU), and what they come to at the ends of the range of positions."""
import ctypes as C
from fractions import Fraction

import numpy as np
import pytest

from paper_2505_04021_amd import binding

BITS = 400


def pi_scaled():
    """pi in 2^-BITS, by Machin's formula."""
    def arctan_of_inverse(x):
        term = total = (1 << (BITS + 64)) // x
        k, sign = 1, -1
        while term:
            term //= x * x
            k += 2
            total += sign * (term // k)
            sign = -sign
        return total
    return 4 * (4 * arctan_of_inverse(5) - arctan_of_inverse(239)) >> 64


CIRCLE = Fraction(2 * pi_scaled(), 1 << BITS)


def some_frequencies():
    rng = np.random.default_rng(3)
    f = [0.0, 1.0, 0.5, 6.283185307179586, 3.141592653589793, 100.25, 1e4, 2.0 ** 32, 2.0 ** 32 - 0.5, 1e-30, 5e-324, 2.0 ** -64, 2.0 ** -62, 1e300 * 1e-300]
    f += [10000.0 ** (-2.0 * i / 128) for i in range(64)] + [500000.0 ** (-2.0 * i / 128) for i in range(64)]
    f += [float(x) for x in rng.uniform(0, 1, 200)] + [float(2.0 ** x) for x in rng.uniform(-80, 32, 200)]
    return f + [-x for x in f]


def test_fractions_are_the_nearest():
    lib = binding._load()
    for f in some_frequencies():
        exact = Fraction(f) / CIRCLE
        got = Fraction(lib.pkv_debug_circle_fraction(f), 1 << 64)
        off = (got - exact) % 1
        off = min(off, 1 - off) * (1 << 64)
        # half a unit, and what the constant's 128 bits leave of frequencies up to 2^32: 2^32 * 2^-131 in units of 2^-64
        assert off <= Fraction(1, 2) + Fraction(1, 1 << 34), (f, float(off))


@pytest.mark.parametrize("pos", [2 ** 31 - 1, -2 ** 31, 2 ** 31 - 12345, 1 << 20, -7])
def test_angles_at_far_positions(pos):
    """What the kernels make of a fraction, (position * fraction) >> 32 modulo 2^32, is within 2^-31 of a circle."""
    lib = binding._load()
    for f in some_frequencies():
        at = (pos * lib.pkv_debug_circle_fraction(f) >> 32) % (1 << 32)
        off = (Fraction(at, 1 << 32) - pos * Fraction(f) / CIRCLE) % 1
        assert min(off, 1 - off) <= Fraction(1, 1 << 31), (f, float(min(off, 1 - off) * 2 ** 32))


def test_frequencies_without_a_meaning_are_refused():
    lib = binding._load()
    f = (C.c_double * 2)(1.0, 0.5)
    for bad in (2.0 ** 64, -2.0 ** 64, 1e300, float("inf"), float("nan")):
        f[1] = bad
        assert lib.rotary_create(4, 0, f, 1.0) == -1, bad

"""Scalings of rotary frequencies that leave the range of doubles are refused, and nothing is written (CPU)."""
import ctypes as C

import pytest

from paper_2505_04021_amd import binding

# rot_dim, base, scaling, factor, trained, low, high
CASES = [(4, 1e300, 2, 1e20, 1, 1, 4), (64, 1e308, 2, 100.0, 1, 1, 4), (64, 1e4, 1, 1e-320, 1, 1, 4), (64, 1e4, 3, 1e-320, 4096.0, 1, 4),
         (64, 1e4, 3, 8.0, 1.7e308, -1e308, 1e308)]


@pytest.mark.parametrize("case", CASES)
def test_refused(case):
    out = (C.c_double * 64)(*([7.0] * 64))
    assert binding._load().rotary_frequencies(*case, out) == -1
    assert list(out) == [7.0] * 64


def test_near_the_border():
    """The largest base that is left, and factors whose frequencies are small, are no fault."""
    lib, out = binding._load(), (C.c_double * 64)()
    assert lib.rotary_frequencies(4, 1e150, 2, 1e70, 1, 1, 4, out) == 2 and list(out[:2]) == [1.0, pytest.approx(1e-145, rel=1e-13)]
    assert lib.rotary_frequencies(4, 1e4, 1, 1e308, 1, 1, 4, out) == 2 and list(out[:2]) == [1e-308, pytest.approx(1e-310, rel=1e-13)]

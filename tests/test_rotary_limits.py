"""Frequencies and magnitudes at the ends of their types, on the host."""
import ctypes
import math

import pytest

import paper_2407_11550_amd as adakv


def test_frequencies_beyond_64_bits_are_refused(lib):
    """base^(-2i/dims) passes 2^1024 for the smallest bases: refused, with nothing written.  Down to 2^-1024 it stays a number."""
    out = (ctypes.c_double * 64)(*([7.0] * 64))
    for scaling, factor in ((0, 1.0), (1, 4.0), (3, 4.0)):
        assert lib.adakv_rotary_frequencies(128, 2.0 ** -1074, scaling, factor, 100, 1.0, 4.0, out) == -1
        assert list(out) == [7.0] * 64
    assert lib.adakv_rotary_frequencies(128, 2.0 ** -1024, 0, 1.0, 0, 0.0, 1.0, out) == 0
    assert all(math.isfinite(f) for f in out) and out[63] == 2.0 ** 1008
    assert lib.adakv_rotary_frequencies(2, 2.0 ** -1074, 0, 1.0, 0, 0.0, 1.0, out) == 0 and out[0] == 1.0


@pytest.mark.parametrize("magnitude", [1e-46, 2.0 ** -150, 5e-324])
def test_a_magnitude_that_fp32_rounds_to_0(lib, magnitude):
    """0 means 1 to the library: such a magnitude is no 1."""
    with pytest.raises(ValueError, match="magnitude"):
        adakv.Rotary(0, magnitude=magnitude, device="cpu")
    assert adakv.Rotary(0, magnitude=2.0 ** -149, device="cpu").c.magnitude > 0

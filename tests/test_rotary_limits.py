"""Frequencies at the ends of their types, on the host."""
import ctypes
import math


def test_frequencies_beyond_64_bits_are_refused(lib):
    """base^(-2i/dims) passes 2^1024 for the smallest bases: refused, with nothing written.  Down to 2^-1024 it stays a number."""
    out = (ctypes.c_double * 64)(*([7.0] * 64))
    for scaling, factor in ((0, 1.0), (1, 4.0), (3, 4.0)):
        assert lib.adakv_rotary_frequencies(128, 2.0 ** -1074, scaling, factor, 100, 1.0, 4.0, out) == -1
        assert list(out) == [7.0] * 64
    assert lib.adakv_rotary_frequencies(128, 2.0 ** -1024, 0, 1.0, 0, 0.0, 1.0, out) == 0
    assert all(math.isfinite(f) for f in out) and out[63] == 2.0 ** 1008
    assert lib.adakv_rotary_frequencies(2, 2.0 ** -1074, 0, 1.0, 0, 0.0, 1.0, out) == 0 and out[0] == 1.0

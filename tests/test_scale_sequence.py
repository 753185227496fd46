"""The kernels around the GEMMs form a unit's scale and its quotients without IEEE
divisions.  These CPU tests run that arithmetic over every mantissa (it does not depend
on the exponent within the normal range, which starts at amax 2^-64 there) from every
value that the hardware's reciprocal, good to an ulp, may give."""
import ctypes

import pytest

from _cbuild import helper


@pytest.fixture(scope="module")
def lib():
    h = helper("scale_sweep")
    for n, a in (("scale_sweep", [ctypes.c_float, ctypes.c_uint32]), ("reciprocal_sweep", [ctypes.c_void_p]),
                 ("last_scale_sweep", [ctypes.c_void_p]), ("quotient_sweep", [ctypes.c_uint64] * 2)):
        getattr(h, n).argtypes, getattr(h, n).restype = a, ctypes.c_uint64
    return h


@pytest.mark.parametrize("fmax", [448.0, 57344.0])
def test_scales_of_every_mantissa(lib, fmax):
    """At the smallest amax that takes this path, around 1 and at the largest finite ones."""
    for exponent in (127 - 64, 126, 127, 254):
        assert lib.scale_sweep(fmax, exponent) == 0, exponent


def test_reciprocals_of_every_mantissa(lib):
    """The refined reciprocal is the correctly rounded one, but for the last mantissa."""
    last = ctypes.c_uint32()
    bad = lib.reciprocal_sweep(ctypes.byref(last))
    assert bad == 0 or (bad == 1 and last.value == 0x7FFFFF)


def test_quotients_by_the_last_mantissa(lib):
    """There the quotient of a power of two alone is off, by a unit in the last place: a
    code is the same on either side, being no middle between two."""
    worst = ctypes.c_uint32(1)
    bad = lib.last_scale_sweep(ctypes.byref(worst))
    assert bad == 0 or (bad == 1 and worst.value == 0)


def test_quotients(lib):
    """With the correctly rounded reciprocal, the residual step gives the correctly
    rounded quotient."""
    assert lib.quotient_sweep(1 << 27, 11) == 0

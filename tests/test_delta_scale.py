"""Scales of the delta rule's state (csrc/delta_scale.h), compiled for the host: powers of two that floats hold, whatever a column
has been, decays to and gets."""
import ctypes as C
import math
import os

import numpy as np
import pytest

from paper_2101_05453_amd import build as libbuild

UP, TOP, KEYS = 120, 11, 2  # the state is brought to 2^11 .. 2^12; what is added comes times keys of 2^2 and more


@pytest.fixture(scope="module")
def hm():
    if not os.path.exists(libbuild.HOSTMATH_LIB):
        libbuild.build_hostmath()
    L = C.CDLL(libbuild.HOSTMATH_LIB)
    L.hm_delta_next_exponent.argtypes = [C.c_int32, C.c_uint32, C.c_uint32]
    L.hm_delta_scaled_whole.argtypes = [C.c_float, C.c_int32]
    L.hm_delta_scaled_whole.restype = L.hm_power_of_two.restype = C.c_float
    return L


def value(bits):
    return float(np.array([bits], np.uint32).view(np.float32)[0])


# every exponent, with the least and the largest mantissa, subnormal numbers and nothing
BITS = [0, 1, 0x7fffff] + [e << 23 | m for e in range(1, 255) for m in (0, 0x7fffff)]


def check(hm, e, kept, added):
    n = hm.hm_delta_next_exponent(e, kept, added)
    assert -UP <= n <= UP
    if kept or added:
        # the larger one in the column's scale, then in the new one; where the scale is at its end it is on that side
        most = max(value(kept), math.ldexp(value(added), e + KEYS))
        new = math.ldexp(most, n - e)
        normal = value(kept) >= 2.0 ** -126 and added == 0 or value(added) >= 2.0 ** -126 and kept == 0
        assert new < 2 ** (TOP + 1) or n == -UP
        assert new >= 2 ** TOP or n == UP or not normal
    return n


def test_every_scale_of_one_number(hm):
    for e in range(-UP, UP + 1):
        for b in BITS:
            n = check(hm, e, b, 0)
            by = hm.hm_power_of_two(min(n - e, 126))  # what a column is brought by before a chunk
            # at n = -UP the scale can only have come down or stayed, and a float times that is a float
            assert by > 0 and (by <= 1 if n == -UP else np.float32(value(b)) * np.float32(by) < 2 ** (TOP + 1))
            check(hm, e, 0, b)


def test_every_scale_of_two_numbers(hm):
    some = BITS[:3] + BITS[3::37]
    for e in range(-UP, UP + 1, 3):
        for kept in some:
            for added in some:
                check(hm, e, kept, added)


def test_what_is_kept_at_the_new_scale_is_a_float(hm):
    rng = np.random.default_rng(0)
    wholes = [0.0, 2.0 ** -149, 2.0 ** -126, 0.5, 1.0] + [math.exp(-x) for x in rng.uniform(0, 110, 60)]
    mosts = [0.0, 2.0 ** -149, 16.0, 2.0 ** 15] + [2.0 ** x for x in rng.uniform(4, 15, 6)]
    for e in range(-UP, UP + 1, 5):
        for whole in wholes:
            for most in mosts:
                w, m = np.float32(whole), np.float32(most)
                kept = m * w
                for added in [0.0, 2.0 ** -149] + [2.0 ** x for x in rng.uniform(-126, 127, 4)]:
                    a = np.float32(added)
                    if kept == 0 and a == 0:
                        continue
                    n = check(hm, e, int(kept.view(np.uint32)), int(a.view(np.uint32)))
                    keep = np.float32(hm.hm_delta_scaled_whole(w, n - e))
                    # at n = -UP what is kept is m times a decay and no more than one
                    assert 0 <= m * keep < (2 ** 15 + 1 if n == -UP else 2 ** (TOP + 2))
                    assert a * np.float32(hm.hm_power_of_two(n)) < 2 ** (TOP + 1 - KEYS)


@pytest.mark.parametrize("keys, top", [(0, 14), (1, 2)])
def test_scales_of_operands(hm, keys, top):
    out = (C.c_float * 2)()
    for b in BITS + [0x7f800000, 0x7fc00000]:  # infinity and NaN too
        hm.hm_delta_scale(b, keys, out)
        up, down = out
        assert up * down == 1 and math.frexp(up)[0] == 0.5 and 2.0 ** -126 <= min(up, down)
        x = np.float32(value(b)) * np.float32(up)
        if value(b) < 2.0 ** 128:  # not infinity, not NaN: fp16 holds it, and it is where it should be
            assert x < 2 ** (top + 1) <= 2 ** 15 and (x >= 2 ** top or value(b) < 2.0 ** (top - 126))

"""Host side of the rotated Append: frequencies in fractions of a turn, and refusals that need no device."""
import ctypes as C
from fractions import Fraction

import numpy as np
import pytest

import paper_2608_23834_b200 as M

# pi to 60 digits
PI = Fraction("3.14159265358979323846264338327950288419716939937510582097494")


def test_turns_are_the_frequencies_in_64_bit_fractions_of_a_turn():
    f = np.concatenate([1e4 ** (-np.arange(64) / 64), 5e5 ** (-np.arange(128) / 128), [0.0, 7.5, -0.25, 1e-9]])
    got = M.mkv_rotary_turns(f)
    for x, t in zip(f, got):
        want = Fraction(float(x)) / (2 * PI) % 1 * 2 ** 64
        # long double holds 64 bits: a unit or two of the last place, times the whole turns taken off
        assert min(abs(int(t) - want), 2 ** 64 - abs(int(t) - want)) <= 2 + 2 * abs(x), (x, t)


def test_an_angle_stays_exact_where_fp32_loses_it():
    f = np.array([1.0, 0.83, 1e-3])
    turns = M.mkv_rotary_turns(f)
    for p in (0, 1, 131071, 10 ** 6, (1 << 31) - 1, -5):
        for x, t in zip(f, turns):
            got = Fraction((p * int(t)) % 2 ** 64, 2 ** 64)
            want = Fraction(float(x)) * p / (2 * PI) % 1
            d = abs(got - want)
            assert min(d, 1 - d) < Fraction(1, 2 ** 31)


def test_bad_frequencies_are_refused():
    for bad in ([float("nan")], [float("inf")], [1.0, -float("inf")]):
        with pytest.raises(M.MkvError) as e:
            M.mkv_rotary_turns(bad)
        assert e.value.code == M.E_INVALID
    assert M.lib().mkv_rotary_turns(None, 3, None) == M.E_INVALID
    assert M.lib().mkv_rotary_turns(None, 0, None) == M.OK
    for kw in (dict(inv_freq=np.ones(7)), dict(inv_freq=np.ones((2, 8))), dict(inv_freq=np.ones(8), axes=np.zeros(4, int)),
               dict(inv_freq=np.ones(8), axes=-np.ones(8, int)), dict(inv_freq=np.ones(8), mscale=float("nan"))):
        with pytest.raises(AssertionError):
            M.Rotary(device="cpu", **kw)


def test_a_bookkeeping_pool_takes_no_tokens():
    hp = M.HostPool(128, 2, 8, 4, 4)
    r = M.Rotary(np.ones(64), device="cpu")
    f = M.lib().mkv_append_rotary
    assert f(hp.handle, None, 0, None, 0, None, 0, None, None, 1, C.byref(r.struct), None, 0, None) == M.E_INVALID
    assert f(None, None, 0, None, 0, None, 0, None, None, 1, C.byref(r.struct), None, 0, None) == M.E_INVALID
    hp.close()

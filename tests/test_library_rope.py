"""The rotation's turns per position on the CPU: the library's host code linked
with stand-ins for the kernels (stub_launches.cpp), against exact integers."""

import ctypes
import math
import random
from fractions import Fraction

import pytest

import paper_2512_20968_amd as ma

from helpers import cache_host_library, turns_per_radian


@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    lib = cache_host_library(tmp_path_factory.mktemp("rope"))
    return lib or pytest.skip("g++ not available")


def turns(lib, freq):
    """The kernel's turn per position of every frequency, in 2^-64 turns."""
    freq = list(freq)
    n = -(-len(freq) // 8) * 8
    r = ma.Rope.make(dict(head_dim=256, rotary_dim=2 * n,
                          inv_freq=freq + [0.0] * (n - len(freq))))
    at = 0x10000
    assert lib.mesh_attn_rope(r, 1, at, 1, at, 256, at, 256, 0, None, 0, None,
                              0, 0, 0, None) == 0
    out = (ctypes.c_uint64 * 128)()
    lib.stub_turns(out)
    return list(out)[:len(freq)]


def check(lib, freq):
    """Rounded to the nearest of 64 bits: half a unit (and the 2^-32 that a cut
    constant may cost), so that position 2^31 is off by 2^-34 of a turn."""
    for f, got in zip(freq, turns(lib, freq)):
        want = Fraction(f) * turns_per_radian() * 2**64
        off = (got - want) % 2**64
        off = min(off, 2**64 - off)
        assert off <= Fraction(1, 2) + Fraction(1, 2**32), (f, float(off))


def test_turns_of_usual_frequencies(lib):
    check(lib, [10000.0 ** (-i / 64) for i in range(64)])
    check(lib, [500000.0 ** (-i / 128) for i in range(128)])


def test_turns_of_every_magnitude(lib):
    """Up to the limit of 2^31 radians, whole turns, subnormals, both signs."""
    far = [6.5, 7.5, 1e2, 1e3, 1e6, 1.2e8, 2.0**30, 2.0**31 - 1,
           math.nextafter(2.0**31, 0.0)]
    near = [0.0, 5e-324, 1e-300, 2.0**-64, 2.0**-63, 2.0**-62, 1e-9, 0.25, 1.0,
            math.pi, 2 * math.pi, math.nextafter(2 * math.pi, 0.0)]
    check(lib, far + near)
    check(lib, [-x for x in far + near])
    rng = random.Random(1)
    check(lib, [rng.choice((-1, 1)) * rng.uniform(0.5, 1.0)
                * 2.0 ** rng.randint(-80, 31) for _ in range(128)])


def test_turns_of_opposite_frequencies_cancel(lib):
    freq = [0.0, 1.0, 7.5, 1e8, 1e-12]
    for a, b in zip(turns(lib, freq), turns(lib, [-f for f in freq])):
        assert (a + b) % 2**64 == 0

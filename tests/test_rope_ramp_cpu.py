"""Host-only checks of LRQK_ROPE_RAMP where the ramp ends behind the last pair.

The ramp runs over pair numbers, from the pair that turns `high` times in l_orig (rounded down) to the one that turns `low` times
(rounded up): j(n) = rot ln(l_orig / (2 pi n)) / (2 ln base).  With a long l_orig or a small base the second is no pair of this rope (they
end at rot/2 - 1), and the pairs there are only have a part of the ramp: all of them turn more than `low` times.  The ends below are worked
out by hand from that formula."""
import math

import numpy as np
import pytest

from test_pages_cpu import lib  # noqa: F401

# rot, base, l_orig, low, high, factor: first and last pair of the ramp
ENDS = [
    ((128, 1e4, 131072, 1.0, 32.0, 4.0), (45, 70)),     # 45.03, 69.11
    ((128, 1e4, 65536, 1.0, 32.0, 4.0), (40, 65)),      # 40.21, 64.29
    ((64, 1e4, 65536, 1.0, 32.0, 4.0), (20, 33)),       # 20.11, 32.15
    ((8, 10.0, 600, 1.0, 32.0, 2.0), (1, 7)),           # 1.90, 7.92: no further than rot - 1
    ((4, 5e5, 8192, 1.0, 4.0, 8.0), (0, 2)),            # 0.88, 1.09
    ((128, 1e4, 32768, 1.0, 32.0, 4.0), (35, 60)),      # 35.39, 59.48: within the pairs
]


def made(lib, rot, base, l_orig, low, high, factor):  # noqa: F811
    turns, _ = lib.lrqk_rope_turns(rot, lib.LRQK_ROPE_RAMP, base=base, factor=factor, low=low, high=high, l_orig=l_orig)
    return np.array([(int(x) & (1 << 64) - 1) / 2.0 ** 64 for x in turns])


@pytest.mark.parametrize("kw,ends", ENDS)
def test_frequencies_by_hand(lib, kw, ends):  # noqa: F811
    rot, base, _, _, _, factor = kw
    first, last = ends
    want = []
    for j in range(rot // 2):
        f, s = base ** (-2 * j / rot), min(max(1 - (j - first) / (last - first), 0.0), 1.0)
        want.append(f * (s + (1 - s) / factor) / (2 * math.pi))
    want = np.array(want)
    # (float64 here: a power and five more roundings)
    assert (np.abs(made(lib, *kw) - want) <= 2.0 ** -48 * want + 2.0 ** -64).all()


@pytest.mark.parametrize("kw,ends", ENDS)
def test_a_pair_that_turns_more_than_low_times_is_not_stretched_fully(lib, kw, ends):  # noqa: F811
    rot, base, l_orig, low, high, factor = kw
    got = made(lib, *kw)
    for j in range(rot // 2):
        plain = base ** (-2 * j / rot) / (2 * math.pi)
        if l_orig * plain > low:
            assert got[j] > plain / factor * (1 + 1e-6), j
        if l_orig * plain > high * base ** (2 / rot):    # in front of the rounded-down end
            assert abs(got[j] - plain) <= 2.0 ** -40 * plain, j


def test_no_ramp_within_the_pairs(lib):  # noqa: F811
    """Both ends behind the last pair: every pair turns more than `high` times and stays; both in front of the first: all but the first
    (where the ramp begins) are stretched."""
    plain = np.array([2.0 ** (-j / 4) for j in range(4)]) / (2 * math.pi)
    assert np.allclose(made(lib, 8, 2.0, 1 << 20, 1.0, 2.0, 4.0), plain, rtol=2.0 ** -40, atol=0)
    plain = np.array([1e4 ** (-j / 4) for j in range(4)]) / (2 * math.pi)
    assert np.allclose(made(lib, 8, 1e4, 1, 1.0, 2.0, 4.0), plain / [1, 4, 4, 4], rtol=2.0 ** -40, atol=0)

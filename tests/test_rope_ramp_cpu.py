"""DKV_ROPE_RAMP where the band reaches past a head's pairs: the first index is cut
at 0 and the last at rot_dim - 1 before the slope is taken."""

import math

import pytest
import torch

import paper_2609_32663_amd as d


def ramp(rot, base, factor, length, low, high):
    at = lambda t: rot * math.log(length / (2 * math.pi * t)) / (2 * math.log(base))  # noqa: E731
    first, last = max(math.floor(at(high)), 0), min(math.ceil(at(low)), rot - 1)
    f = []
    for i in range(rot // 2):
        if last > first:
            keep = min(max(1.0 - (i - first) / (last - first), 0.0), 1.0)
        else:  # nothing between them
            keep = 1.0 if i <= last else 0.0
        p = base ** (-2.0 * i / rot)
        f.append(keep * p + (1.0 - keep) * p / factor)
    return torch.tensor(f, dtype=torch.float64)


# (rot_dim, base, factor, trained_len, low, high, index of the first pair before its cut, of the last)
CASES = [(64, 1e4, 4.0, 128.0, 1.0, 32.0, -2, 11),       # a small model's length: the fastest pair turns 20 times
         (128, 5e5, 8.0, 150.0, 1.0, 32.0, -2, 16),
         (64, 1e4, 4.0, 8192.0, 1.0, 32.0, 12, 25),      # the band within the pairs
         (16, 2.0, 4.0, 1e6, 1.0, 32.0, 98, 139),        # beyond the last index on both sides
         (16, 4.0, 4.0, 3000.0, 0.05, 32.0, 15, 53),
         (16, 4.0, 4.0, 600.0, 0.05, 32.0, 6, 44),       # the last index beyond
         (64, 1e4, 4.0, 6.0, 1.0, 4.0, -5, 0),           # only the fastest pair is left
         (64, 1e4, 4.0, 3.0, 1.0, 4.0, -8, -2)]          # none turns once


@pytest.mark.parametrize("rot, base, factor, length, low, high, first, last", CASES)
def test_ramp_within_the_pairs(rot, base, factor, length, low, high, first, last):
    at = lambda t: rot * math.log(length / (2 * math.pi * t)) / (2 * math.log(base))  # noqa: E731
    assert (math.floor(at(high)), math.ceil(at(low))) == (first, last)
    f, m = d.dkv_rope_freqs(d.DKV_ROPE_RAMP, rot, base, factor, length, low, high)
    want = ramp(rot, base, factor, length, low, high)
    # one rounding to fp32, and the double's own on either side
    assert ((f.double() / want - 1).abs() <= 2.0 ** -24 * (1 + 2.0 ** -20)).all(), f.double() / want - 1
    assert abs(m - (0.1 * math.log(factor) + 1.0)) < 2.0 ** -22


def test_the_fastest_pair_of_a_short_length_stays():
    f, _ = d.dkv_rope_freqs(d.DKV_ROPE_RAMP, 64, 1e4, 4.0, 128.0, 1.0, 32.0)
    assert f[0] == 1.0

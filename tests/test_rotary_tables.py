"""Frequencies of the rotary positions, pair by pair, from the scalings' formulas. Host code only."""
import math

import pytest
import torch

import paper_2604_11288_b200 as ta
from paper_2604_11288_b200 import build as ta_build


@pytest.fixture(scope="module", autouse=True)
def lib():
    ta_build.build()


def _table(d_rot, base, kind, factor, orig, low, high):
    phase = torch.empty(d_rot // 2, dtype=torch.int64)
    magnitude = ta.ta_rotary_table(d_rot, base, kind, factor, orig, low, high, phase)
    turns = [(int(p) % 2 ** 64) / 2.0 ** 64 for p in phase]
    return magnitude, torch.tensor(turns, dtype=torch.float64) * 2 * math.pi


def _close(got, want):
    # two roundings of pow and one each of the weight's operations in 64 bits; turns are whole multiples of 2^-64
    assert ((got - want).abs() <= 1e-11 * want + 2 * math.pi * 2.0 ** -64).all(), (got / want - 1).abs().max()


@pytest.mark.parametrize("d_rot,base,factor,orig", [(128, 500000.0, 8.0, 8192.0), (128, 10000.0, 32.0, 4096.0), (64, 1e6, 4.0, 32768.0),
                                                    (8, 10000.0, 2.0, 2048.0), (128, 150000.0, 1.0, 4096.0)])
@pytest.mark.parametrize("low,high", [(1.0, 32.0), (1.0, 4.0), (0.5, 1000.0)])
def test_every_pair(d_rot, base, factor, orig, low, high):
    i = torch.arange(d_rot // 2, dtype=torch.float64)
    f = base ** (-2.0 * i / d_rot)
    turns = orig * f / (2 * math.pi)
    # pairs by index: the index at which a pair turns r times within the original length, rounded outwards and kept in the head
    index = (lambda r: d_rot * math.log(orig / (r * 2 * math.pi)) / (2 * math.log(base)))
    first, last = max(math.floor(index(high)), 0), min(math.ceil(index(low)), d_rot - 1)
    by_index = 1.0 - ((i - first) / max(last - first, 0.001)).clamp(0.0, 1.0)
    by_turns = ((turns - low) / (high - low)).clamp(0.0, 1.0)
    want = {ta.TA_SCALING_PLAIN: f, ta.TA_SCALING_LINEAR: f / factor,
            ta.TA_SCALING_BASE: (base * factor ** (d_rot / (d_rot - 2))) ** (-2.0 * i / d_rot),
            ta.TA_SCALING_RAMP: by_index * f + (1.0 - by_index) * f / factor,
            ta.TA_SCALING_BAND: by_turns * f + (1.0 - by_turns) * f / factor}
    for kind, w in want.items():
        magnitude, got = _table(d_rot, base, kind, factor, orig, low, high)
        _close(got, w)
        assert abs(magnitude - (0.1 * math.log(factor) + 1.0 if kind == ta.TA_SCALING_RAMP else 1.0)) < 1e-6
    if d_rot == 128 and factor > 1 and last < d_rot // 2:
        inside = (i > first) & (i < last)
        assert inside.sum() > 1 and (want[ta.TA_SCALING_RAMP] < f)[inside].all() and (want[ta.TA_SCALING_RAMP] > f / factor)[inside].all()

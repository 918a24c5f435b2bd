"""Types that the descriptions of caches and rotations insist on: what is described reaches the kernels as an address."""
import numpy as np
import pytest
import torch

import paper_2604_11288_b200 as ta


def _rows(dtype):
    return torch.zeros(1, 6, 2, 16, 128).to(dtype)


@pytest.mark.parametrize("what", ["table", "lens", "lens per unit"])
@pytest.mark.parametrize("dtype", [torch.int64, torch.int16, torch.float32])
def test_tables_and_lengths_are_int32(what, dtype):
    shape = {"table": (2, 3), "lens": (2,), "lens per unit": (1, 2, 2)}[what]
    kw = dict(table=torch.zeros(2, 3, dtype=torch.int32))
    k = _rows(torch.bfloat16)
    ta.make_cache(k, k, **{**kw, what.split()[0]: torch.zeros(shape, dtype=torch.int32)})
    with pytest.raises(AssertionError, match="int32"):
        ta.make_cache(k, k, **{**kw, what.split()[0]: torch.zeros(shape, dtype=dtype)})


@pytest.mark.parametrize("dtype", [torch.int8, torch.float8_e4m3fn])
def test_scales_are_float32_and_go_with_8_bits(dtype):
    k, s = _rows(dtype), torch.zeros(1, 6, 2, 16)
    ta.make_cache(k, k, s, s, batch=2)
    for a, b in ((s.half(), s.half()), (s, s.bfloat16()), (s.double(), s), (None, None), (s, None), (None, s), (s, s[:, :5])):
        with pytest.raises(AssertionError, match="scale"):
            ta.make_cache(k, k, a, b, batch=2)
    k = _rows(torch.bfloat16)
    for a, b in ((s, s), (s, None), (None, s)):
        with pytest.raises(AssertionError, match="scale"):
            ta.make_cache(k, k, a, b, batch=2)


def test_frequencies_and_positions():
    for phase in (torch.zeros(64, dtype=torch.int64), torch.zeros(64, dtype=torch.uint64), np.zeros(64, dtype=np.uint64)):
        assert ta.ta_rotary_table(128, 10000.0, ta.TA_SCALING_PLAIN, 1.0, 0.0, 0.0, 0.0, phase) == 1.0
        assert ta.make_rotary(phase, 128, positions=torch.zeros(3, dtype=torch.int32)).d_rot == 128
    for phase in (torch.zeros(63, dtype=torch.int64), torch.zeros(64, dtype=torch.float32), torch.zeros(64, dtype=torch.float64),
                  torch.zeros(128, dtype=torch.int64)[::2], np.zeros(64, dtype=np.uint32), np.zeros(63, dtype=np.uint64)):
        with pytest.raises(AssertionError, match="64-bit"):
            ta.ta_rotary_table(128, 10000.0, ta.TA_SCALING_PLAIN, 1.0, 0.0, 0.0, 0.0, phase)
    with pytest.raises(AssertionError, match="64-bit"):
        ta.make_rotary(torch.zeros(64), 128)
    with pytest.raises(AssertionError, match="int32"):
        ta.make_rotary(torch.zeros(64, dtype=torch.int64), 128, positions=torch.zeros(3, dtype=torch.int64))

"""The scratch of the attention of new tokens: what a context is told to bring is enough for every smaller call too. How a call is
cut is host code, compiled here by itself."""
import ctypes
import itertools
import os
import random
import subprocess

import pytest
import torch

import paper_2604_11288_b200 as ta
from paper_2604_11288_b200 import build as ta_build

SOURCE = r"""
#include "ta_attend_rule.h"
extern "C" long long need(long long units, int rows, int d, int max_len, int codes, int ragged, int mass) {
  return (long long)ta_attend_sizes_of(units, rows, d, max_len, ta_attend_slots(ta_attend_plan_of(units, rows, max_len, codes, ragged), units), mass).all();
}
extern "C" long long told(long long units, int rows, int d, int max_len, int mass) {
  return (long long)ta_attend_sizes_of(units, rows, d, max_len, ta_attend_most_slots(units, rows, max_len), mass).all();
}
extern "C" void plan(long long units, int rows, int max_len, int codes, int ragged, int* out) {
  const ta_attend_plan p = ta_attend_plan_of(units, rows, max_len, codes, ragged);
  out[0] = p.mb, out[1] = p.warps, out[2] = p.row_blocks, out[3] = p.piece, out[4] = p.pieces, out[5] = p.target;
}
"""


@pytest.fixture(scope="module")
def rule(tmp_path_factory):
    d = tmp_path_factory.mktemp("attend_rule")
    (d / "rule.cpp").write_text(SOURCE)
    subprocess.run([os.environ.get("CXX", "g++"), "-std=c++17", "-O1", "-fPIC", "-shared", "-I",
                    os.path.join(os.path.dirname(ta.__file__), "csrc"), str(d / "rule.cpp"), "-o", str(d / "rule.so")], check=True)
    lib = ctypes.CDLL(str(d / "rule.so"))
    for f in (lib.need, lib.told):
        f.restype = ctypes.c_longlong
    ints = [ctypes.c_int] * 5
    lib.need.argtypes, lib.told.argtypes = [ctypes.c_longlong] + ints + [ctypes.c_int], [ctypes.c_longlong] + ints[:4]
    lib.plan.argtypes = [ctypes.c_longlong] + ints[:4] + [ctypes.c_void_p]
    return lib


@pytest.fixture(scope="module")
def lib():
    ta_build.build()
    return ta.binding.lib()


def _cache(batch, layers=1, kv=8, d=128, form=ta.TA_CACHE_BF16):
    k = torch.zeros(1, 1, 1, 1, d, dtype=torch.bfloat16)
    c = ta.make_cache(k, k, batch=1)
    c.n_layers, c.batch, c.Hkv, c.format, c.keep = layers, batch, kv, form, k
    if form != ta.TA_CACHE_BF16:
        c.k_scale = c.v_scale = k.data_ptr()
    return c


@pytest.mark.parametrize("mass", [False, True])
@pytest.mark.parametrize("max_len", [1, 129, 4096, 131072])
def test_a_larger_call_is_told_no_less(lib, max_len, mass):
    said = {}
    for layers, batch, G, T in itertools.product((1, 3, 32), (1, 16, 128, 222, 256), (1, 4, 5), (1, 2, 8, 64)):
        said[layers, batch, G, T] = ta.ta_attend_scratch_bytes(_cache(batch, layers), 8 * G, T, max_len, mass)
        assert ta.ta_attend_scratch_bytes(_cache(batch, layers), 8 * G, T, max(0, max_len - 1), mass) <= said[layers, batch, G, T]
        assert ta.ta_attend_scratch_bytes(_cache(batch, layers, d=64), 8 * G, T, max_len, mass) <= said[layers, batch, G, T]
        assert mass or said[layers, batch, G, T] <= 92e6
    for a, b in itertools.product(said, said):
        assert not all(x <= y for x, y in zip(a, b)) or said[a] <= said[b], (a, b)


def test_enough_for_every_smaller_call(rule):
    # the most that any number of units needs, at the lengths where a piece is added and at a few others
    for rows in (1, 8, 9, 16, 17, 32, 33, 200, 4096):
        for max_len in (0, 1, 128, 129, 256, 257, 1000, 5000, 20000, 131072, 1 << 20):
            for codes, ragged in itertools.product((0, 1), (0, 1, 2, 1024, 1025)):
                most = 0
                for units in itertools.chain(range(1, 500), range(500, 9000, 37), (16384, 16385, 10 ** 6)):
                    most = max(most, rule.need(units, rows, 128, max_len, codes, ragged, 0))
                    assert most <= rule.told(units, rows, 128, max_len, 0), (units, rows, max_len)
    rng = random.Random(1)
    for _ in range(100000):  # and calls that are smaller in several ways
        units, rows, n = (int(2 ** rng.uniform(0, e)) for e in (15, 12, 17))
        u, r, m = (rng.randint(1, x) for x in (units, rows, n))
        mass = rng.randint(0, 1)
        assert rule.need(u, r, rng.choice((64, 128)), m, rng.randint(0, 1), rng.choice((0, 1, 2, 16, 2000)), mass) <= rule.told(units, rows, 128, n, mass)


def test_the_library_tells_what_the_rule_says(rule, lib):
    for batch, G, T, n, mass in ((1, 4, 1, 4096, 0), (16, 4, 4, 131072, 0), (256, 1, 1, 257, 1), (16, 2, 64, 1000, 1)):
        for form in (ta.TA_CACHE_BF16, ta.TA_CACHE_INT8):
            told = ta.ta_attend_scratch_bytes(_cache(batch, form=form), 8 * G, T, n, bool(mass))
            assert 0 <= told - rule.told(8 * batch, G * T, 128, n, mass) <= 512


def test_plans_cover_their_rows(rule):
    out = (ctypes.c_int * 6)()
    for units, rows, max_len, codes, ragged in itertools.product(
            (1, 8, 128, 443, 444, 445, 1775, 1776, 16384, 16385), (1, 8, 9, 16, 17, 100), (0, 1, 128, 129, 257, 5000, 131072), (0, 1), (0, 2, 1025)):
        rule.plan(units, rows, max_len, codes, ragged, out)
        mb, warps, row_blocks, piece, pieces, target = out
        height = 8 if mb == 0 else 16 * mb
        assert row_blocks * height >= rows > (row_blocks - 1) * height
        assert pieces >= 1 and piece % 128 == 0 and pieces * height <= 4096 and (target > 0 or pieces * piece >= max_len)
        assert pieces == 1 or units * row_blocks <= 16384  # a counter each
        assert warps == 4 or (warps == 2 and mb == 0 and pieces == 1)
        assert target == 0 or (pieces > 1 and ragged > 1 and units * row_blocks <= 444)  # (sequences are units too)


def test_more_blocks_than_a_grid_has_are_refused(lib):
    ok = _cache(1 << 20, layers=16)  # 2^27 units
    assert ta.ta_attend_scratch_bytes(ok, 8 * 256, 1, 100) > 0
    for T in (2, 64):
        with pytest.raises(ta.TAError) as e:
            ta.ta_attend_scratch_bytes(ok, 8 * 256, T, 100)
        assert e.value.status == ta.TA_ERR_UNSUPPORTED


def test_the_variants_that_calls_of_these_sizes_take(rule):
    """What the tests of the variants rely on: [query rows of a block / 16, warps, row blocks, piece, pieces, cut on the device]."""
    out = (ctypes.c_int * 6)()

    def plan(*args):
        rule.plan(*args, out)
        return list(out)[:2] + [out[4], out[5] > 0]
    for codes, ragged in itertools.product((0, 1), (0, 75)):
        assert plan(1800, 8, 70, codes, ragged) == [0, 2, 1, False]      # many short units
        assert plan(1920, 4, 65, codes, ragged) == [0, 2, 1, False]
        assert plan(2560, 4, 257, codes, 0) == [0, 2, 1, False]
        assert plan(16408, 8, 150, codes, 2051) == [0, 2, 1, False]      # more row blocks than counters
        assert plan(16408, 16, 150, codes, 2051)[2:] == plan(8240, 64, 150, codes, 1030)[2:] == [1, False]
        for rows in (4, 16, 32):
            assert plan(512, rows, 1100, codes, 64)[2] > 1 and not out[5]  # more units than run at once, in pieces
        assert [plan(b, 4, 400, codes, b)[3] for b in (1, 2, 222, 377, 444, 445)] == [False, True, True, True, False, False]

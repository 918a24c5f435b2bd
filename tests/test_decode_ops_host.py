"""What the decode loop's operators check and compute on the host, without a device, and both ways of marshalling them."""
import ctypes as C

import pytest
import torch

import paper_2604_11288_b200 as ta
from paper_2604_11288_b200 import build as ta_build


@pytest.fixture(scope="module")
def lib():
    ta_build.build()
    return ta.binding.lib()


def _cache(**kw):
    k = torch.zeros(1, 6, 2, 16, 128, dtype=torch.bfloat16)
    c = ta.make_cache(k, k, table=torch.zeros(2, 3, dtype=torch.int32), len_uniform=3)
    c.keep = k
    for n, v in kw.items():
        setattr(c, n, v)
    return c


def test_descriptions_of_caches():
    k = torch.zeros(2, 6, 16, 3, 64, dtype=torch.int8).transpose(2, 3)
    s = torch.zeros(2, 6, 16, 3).transpose(2, 3)
    c = ta.make_cache(k, k, s, s, table=torch.zeros(2, 3, dtype=torch.int32), lens=torch.zeros(2, 2, 3, dtype=torch.int32))
    assert (c.n_layers, c.batch, c.Hkv, c.d, c.page, c.n_pages, c.pages_per_seq) == (2, 2, 3, 64, 16, 6, 3)
    assert (c.format, c.lens_per_unit) == (ta.TA_CACHE_INT8, 1)
    assert (c.stride_l, c.stride_p, c.stride_h, c.stride_r) == (6 * 3 * 16 * 64, 3 * 16 * 64, 64, 3 * 64)
    assert (c.scale_stride_h, c.scale_stride_r) == (1, 3)
    dense = torch.zeros(1, 4, 2, 33, 128, dtype=torch.bfloat16)
    c = ta.make_cache(dense, dense, batch=4)
    assert (c.table, c.pages_per_seq, c.page, c.format) == (None, 1, 33, ta.TA_CACHE_BF16)
    for bad in (lambda: ta.make_cache(dense, dense.float(), batch=4), lambda: ta.make_cache(dense.float(), dense.float(), batch=4),
                lambda: ta.make_cache(dense, dense[..., :16, :], batch=4), lambda: ta.make_cache(dense, dense, batch=3),
                lambda: ta.make_cache(dense, dense, batch=4, lens=torch.zeros(3, dtype=torch.int32))):
        with pytest.raises(AssertionError):
            bad()


def test_scratch_and_its_refusals(lib):
    small, large = ta.ta_attend_scratch_bytes(_cache(), 8, 1, 48), ta.ta_attend_scratch_bytes(_cache(), 8, 1, 48, True)
    assert 0 < small < large
    longer = ta.ta_attend_scratch_bytes(_cache(), 8, 1, 100000)
    assert longer > small  # pieces of a long cache are joined there
    for change, args, status in (
            (dict(k=None), (8, 1, 48), ta.TA_ERR_INVALID_ARG), (dict(format=7), (8, 1, 48), ta.TA_ERR_INVALID_ARG),
            (dict(d=80), (8, 1, 48), ta.TA_ERR_UNSUPPORTED), (dict(stride_p=4), (8, 1, 48), ta.TA_ERR_ALIGNMENT),
            (dict(stride_r=64), (8, 1, 48), ta.TA_ERR_INVALID_ARG), (dict(format=ta.TA_CACHE_INT8), (8, 1, 48), ta.TA_ERR_INVALID_ARG),
            (dict(n_pages=1 << 30, stride_p=1 << 20), (8, 1, 48), ta.TA_ERR_UNSUPPORTED),
            ({}, (7, 1, 48), ta.TA_ERR_INVALID_ARG), ({}, (8, 0, 48), ta.TA_ERR_INVALID_ARG), ({}, (8, 65, 48), ta.TA_ERR_UNSUPPORTED),
            ({}, (8, 1, -1), ta.TA_ERR_INVALID_ARG), ({}, (8, 1, (1 << 20) + 1), ta.TA_ERR_UNSUPPORTED),
            ({}, (2 * 257, 1, 48), ta.TA_ERR_UNSUPPORTED)):
        with pytest.raises(ta.TAError) as e:
            ta.ta_attend_scratch_bytes(_cache(**change), *args)
        assert e.value.status == status, (change, args)


def test_both_marshallings_refuse_alike(lib):
    batch, view, cache = ta.make_batch(1, 2, 1, 1, 2), ta.ta_bf16_view(), _cache()
    rot = ta.make_rotary(None, 128)
    native, plain = ta.binding._native(), ta.binding._CtypesCalls(lib)
    for c in (native, plain):
        for r in (None, rot):
            assert [c.ta_rotate(None, batch, 8, 2, 128, r, view, view, view, view, None),
                    c.ta_cache_append(None, cache, batch, r, view, view, None, None),
                    c.ta_cache_read(None, cache, batch, None, view, view, None),
                    c.ta_attend(None, cache, 8, 1, 0, 48, True, 0.0, r, view, view, None, None, 0, None)] == [ta.TA_ERR_INVALID_ARG] * 4
    assert C.sizeof(ta.ta_cache) == 4 * 8 + 8 * 8 + 2 * 8 + 10 * 4 and C.sizeof(ta.ta_rotary) == 2 * 8 + 4 * 4


def test_rotary_table_needs_no_device(lib):
    phase = torch.empty(4, dtype=torch.int64)
    assert ta.ta_rotary_table(8, 10000.0, ta.TA_SCALING_LINEAR, 2.0, 0.0, 0.0, 0.0, phase) == 1.0
    turns = phase.double() / 2.0 ** 64
    want = torch.tensor([10000.0 ** (-i / 4) / 2 / 6.283185307179586 for i in range(4)], dtype=torch.float64)
    assert torch.allclose(turns, want, rtol=1e-12, atol=2.0 ** -63)
    with pytest.raises(ta.TAError):
        ta.ta_rotary_table(8, 0.5, ta.TA_SCALING_PLAIN, 1.0, 0.0, 0.0, 0.0, phase)

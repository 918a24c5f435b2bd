"""Attention calls at the ends of what a call may be, and one context for calls of many sizes."""
import pytest
import torch

import paper_2604_11288_b200 as ta
from decode_testlib import DEV, Cache, Ctx, run_attend

pytestmark = pytest.mark.gpu


def _q(B, H, T, d=128, seed=0):
    g = torch.Generator().manual_seed(seed + 100)
    return torch.randn((1, B, H, T, d), generator=g).to(torch.bfloat16)


@pytest.mark.parametrize("form", ["bf16", "int8"])
def test_a_context_for_the_largest_call_is_enough_for_smaller_ones(form):
    n, kv, G = 1000, 8, 2
    large = Cache(1, 256, kv, 128, 250, 4, form, dense=True, len_uniform=n)
    with Ctx(ta.ta_attend_scratch_bytes(large.struct(), kv * G, 1, n)) as h:
        q = _q(256, kv * G, 1).to(DEV)
        run_attend(large, q, 1, max_len=n, with_mass=False, ctx=h)
        for B, most in ((1, n), (5, 700), (7, n), (40, 999), (200, n)):
            c = Cache(1, B, kv, 128, 250, 4, form, dense=True, lens=[most - 3 * b for b in range(B)], seed=B)
            got = run_attend(c, q[:, :B].contiguous(), 1, max_len=most, with_mass=False, ctx=h)
            assert ta.ta_ctx_poll(h) == ta.TA_OK
            want = run_attend(c, q[:, :B].contiguous(), 1, max_len=most, with_mass=False)  # in a context of its own
            assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


@pytest.mark.parametrize("form", ["bf16", "e4m3"])
@pytest.mark.parametrize("stride", [None, 0, 5])
def test_a_largest_length_of_zero(form, stride):
    c, q = Cache(1, 2, 2, 128, 16, 2, form, len_uniform=0), _q(2, 8, 2).to(DEV)
    s, out = c.struct(), torch.full_like(q, 7.0)
    lse, mass = torch.full((1, 2, 8, 2), 7.0, device=DEV), torch.full((64,), 7.0, device=DEV)
    with Ctx(ta.ta_attend_scratch_bytes(s, 8, 2, 0, True)) as h:
        ta.ta_attend(h, s, 8, 2, 0, 0, True, 0.0, None, ta.view(q), ta.view(out), lse, None if stride is None else mass, stride or 0,
                     torch.cuda.current_stream().cuda_stream)
        torch.cuda.synchronize()
        assert ta.ta_ctx_poll(h) == ta.TA_OK
    assert (out == 0).all() and (lse == -torch.inf).all()
    written = 4 * (stride or 0)  # of every sequence and head
    assert (mass[:written] == 0).all() and (mass[written:] == 7.0).all()


def test_more_room_for_the_mass_than_a_grid_is_high():
    stride = 65535 * 1024 + 4
    c, q = Cache(1, 1, 1, 128, 16, 2, lens=[21]), _q(1, 2, 1).to(DEV)
    want = run_attend(c, q, 1)[2]
    mass, out = torch.full((stride + 8,), 7.0, device=DEV), torch.empty_like(q)
    s = c.struct()
    with Ctx(ta.ta_attend_scratch_bytes(s, 2, 1, 32, True)) as h:
        ta.ta_attend(h, s, 2, 1, 0, 32, True, 0.0, None, ta.view(q), ta.view(out), None, mass, stride,
                     torch.cuda.current_stream().cuda_stream)
        torch.cuda.synchronize()
        assert ta.ta_ctx_poll(h) == ta.TA_OK
    assert torch.equal(mass[:32].cpu().double(), want[0, 0, 0]) and int(mass[32:stride].count_nonzero()) == 0
    assert (mass[stride:] == 7.0).all()

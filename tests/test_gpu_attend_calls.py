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

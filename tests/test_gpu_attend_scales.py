"""Attention over 8-bit caches whose value scales lie far apart: no row takes precision from a query that does not see it, or that
gives it next to no probability."""
import pytest
import torch

from decode_testlib import DEV, Cache, attend_reference, codes, run_attend, within

pytestmark = pytest.mark.gpu
FORMS = ["e4m3", "int8"]


def _q(B, H, T, d, seed=0):
    g = torch.Generator().manual_seed(seed + 100)
    return torch.randn((1, B, H, T, d), generator=g).to(torch.bfloat16)


def _at(c, b, row):
    return int(c.page_ids(b)[row // c.page]), row % c.page


@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("times", [1e6, 1e12, 1e30])
@pytest.mark.parametrize("G,T,d", [(4, 2, 128), (4, 4, 128), (4, 7, 128), (2, 4, 64)])
def test_unseen_rows_of_any_finite_scale_have_no_influence(form, times, G, T, d):
    lens = [0, 5, 16, 83, 700]
    q = _q(len(lens), 2 * G, T, d).to(DEV)

    def filled(rows_of):
        c = Cache(1, len(lens), 2, d, 16, 44, form, lens=lens)
        for b, n in enumerate(lens):
            for r in rows_of(b, n, c):
                at, off = _at(c, b, r)
                c.dev["v_scale"][:, at, :, off] *= times
        return run_attend(c, q, T)

    clean = filled(lambda b, n, c: [])
    for a, x in zip(clean, filled(lambda b, n, c: range(n, c.wide * c.page))):  # behind the last row
        assert torch.equal(a, x)
    got = filled(lambda b, n, c: [n - 2] if n >= T else [])  # seen by the last two tokens
    assert torch.equal(got[0][..., :T - 2, :], clean[0][..., :T - 2, :])
    for b, n in enumerate(lens):
        assert n < T or not torch.equal(got[0][:, b, :, T - 2:], clean[0][:, b, :, T - 2:])
    assert torch.equal(got[1], clean[1]) and torch.equal(got[2], clean[2])


@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("times", [1e6, 1e12, 1e20, 1e30])
@pytest.mark.parametrize("G,T", [(4, 1), (4, 4), (4, 8)])
@pytest.mark.parametrize("rows", [[3], [250], [499], list(range(160))])
def test_seen_rows_weigh_as_their_probability_says(form, times, G, T, rows):
    """Rows that every query gives e^-40 to e^-80 of the others' probability, with value scales far above theirs."""
    n, d = 500, 128
    c = Cache(1, 1, 1, d, 16, 32, form, lens=[n])
    base = torch.randn(d, generator=torch.Generator().manual_seed(5))
    q = (base + 0.1 * _q(1, G, T, d).float()).to(torch.bfloat16)
    code, scale = codes((-5.0 * base).to(torch.bfloat16).float().unsqueeze(0), form)
    for r in rows:
        at, off = _at(c, 0, r)
        c.dev["k"].view(torch.int8)[0, at, 0, off] = code[0].view(torch.int8).to(DEV)
        c.dev["k_scale"][0, at, 0, off] = float(scale[0])
        c.dev["v_scale"][0, at, 0, off] *= times
    got = run_attend(c, q.to(DEV), T)
    out, lse, mass, tol, lse_tol, mass_tol = attend_reference(c, q, T)
    within(got[0], out, tol, "out")
    within(got[1], lse, lse_tol, "lse")


@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("T", [1, 4])
def test_the_smallest_scales(form, T):
    c = Cache(1, 1, 1, 128, 16, 20, form, lens=[300])
    c.dev["v_scale"].fill_(2.0 ** -100 / 127.0)
    q = _q(1, 4, T, 128)
    got = run_attend(c, q.to(DEV), T)
    out, lse, mass, tol, lse_tol, mass_tol = attend_reference(c, q, T)
    # attend_reference's tolerance ends at 1e-30, about the size of these values; what is lost below fp32's normal numbers is 2^-150 a
    # probability, times 300 rows and codes of 448
    within(got[0] * 2.0 ** 100, out * 2.0 ** 100, 2.0 ** 100 * (tol - 1e-30) + 2.0 ** -30, "out")


@pytest.mark.parametrize("n", [40, 64, 500])
@pytest.mark.parametrize("T", [1, 3])
def test_a_scale_of_nan_that_is_seen_is_told_in_any_tile(n, T):
    """Whatever its probability: whole tiles and the ones at a sequence's end alike."""
    c = Cache(1, 1, 1, 128, 16, 32, "e4m3", lens=[n])
    base = torch.randn(128, generator=torch.Generator().manual_seed(5))
    q = base.to(torch.bfloat16).expand(1, 1, 2, T, 128).contiguous()
    for r in (1, n - T):  # probabilities of 0 in 32 bits
        code, scale = codes((-9.0 * base).to(torch.bfloat16).float().unsqueeze(0), "e4m3")
        at, off = _at(c, 0, r)
        c.dev["k"].view(torch.int8)[0, at, 0, off] = code[0].view(torch.int8).to(DEV)
        c.dev["k_scale"][0, at, 0, off] = float(scale[0])
        clean = run_attend(c, q.to(DEV), T)
        old = float(c.dev["v_scale"][0, at, 0, off])
        c.dev["v_scale"][0, at, 0, off] = float("nan")
        got = run_attend(c, q.to(DEV), T)
        assert clean[0].isfinite().all() and got[0].isnan().all()
        c.dev["v_scale"][0, at, 0, off] = old

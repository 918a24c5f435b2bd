"""Attention of new tokens over a cache against a 64-bit statement: formats, head groups, lengths, masks, mass, splits."""
import math

import pytest
import torch

import paper_2604_11288_b200 as ta
from decode_testlib import DEV, Cache, Ctx, attend_reference, frequencies, rotary, run_attend, within
from test_gpu_cache import _bad_caches

pytestmark = pytest.mark.gpu


def _q(L, B, H, T, d, seed=0, scale=1.0):
    g = torch.Generator().manual_seed(seed + 100)
    return (torch.randn((L, B, T, H, d), generator=g) * scale).to(torch.bfloat16).transpose(2, 3)


def _check(c, q, T=1, new_rows=0, causal=True, scale=0.0, rot=None, ref_rot=None, **kw):
    got = run_attend(c, q.to(DEV), T, new_rows, causal=causal, scale=scale, rot=rot, **kw)
    out, lse, mass, tol, lse_tol, mass_tol = attend_reference(c, q, T, new_rows, causal, scale, ref_rot)
    within(got[0], out, tol, "out")
    within(got[1], lse, lse_tol, "lse")
    if got[2] is not None:
        n = min(mass.shape[-1], got[2].shape[-1])
        within(got[2][..., :n], mass[..., :n], mass_tol[..., :n], "mass")
        assert (got[2][..., n:] == 0).all()
    return got


LENS = [0, 1, 15, 16, 17, 31, 33, 63, 64, 65, 127, 129, 200, 255, 256, 1000]


@pytest.mark.parametrize("form", ["bf16", "e4m3", "int8"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("kv,G", [(1, 1), (2, 4), (1, 8), (2, 3)])
def test_lengths(form, d, kv, G):
    c = Cache(1, len(LENS), kv, d, 16, 63, form, lens=LENS)
    _check(c, _q(1, len(LENS), kv * G, 1, d))


@pytest.mark.parametrize("form", ["bf16", "int8"])
@pytest.mark.parametrize("T,causal", [(1, True), (2, True), (4, True), (5, False), (7, True), (16, True), (64, True)])
@pytest.mark.parametrize("G", [1, 2, 5])
def test_several_tokens(form, T, causal, G):
    lens = [0, 1, 2, 6, 17, 64, 300]
    c = Cache(1, len(lens), 2, 128, 16, 19, form, "rows", lens=lens)
    _check(c, _q(1, len(lens), 2 * G, T, 128), T, causal=causal)


@pytest.mark.parametrize("G,T", [(16, 1), (24, 1), (33, 1), (64, 2), (256, 1)])
def test_many_heads_of_one_group(G, T):
    c = Cache(1, 2, 1, 128, 16, 20, "e4m3", lens=[300, 77])
    _check(c, _q(1, 2, G, T, 128), T)


@pytest.mark.parametrize("page,order", [(1, "heads"), (3, "rows"), (16, "rows"), (48, "heads"), (128, "rows"), (1024, "heads")])
@pytest.mark.parametrize("form", ["bf16", "e4m3"])
def test_pages(page, order, form):
    lens = [5, 130, 257]
    c = Cache(2, 3, 2, 128, page, -(-260 // page), form, order, lens=lens)
    _check(c, _q(2, 3, 8, 1, 128))


@pytest.mark.parametrize("n", [5000, 20011])
@pytest.mark.parametrize("form,d,T", [("bf16", 128, 1), ("e4m3", 128, 1), ("int8", 64, 3)])
def test_long(n, form, d, T):
    c = Cache(1, 2, 1, d, 64, -(-n // 64), form, lens=[n, n // 3])
    _check(c, _q(1, 2, 4, T, d), T)
    _check(c, _q(1, 2, 4, T, d), T, with_mass=False)


def test_lengths_per_unit_and_layers():
    g = torch.Generator().manual_seed(8)
    L, B, kv = 3, 2, 4
    lens = torch.randint(0, 90, (L, B, kv), generator=g).tolist()
    c = Cache(L, B, kv, 128, 30, 3, "bf16", dense=True, lens=lens)
    _check(c, _q(L, B, 8, 1, 128))
    _check(c, _q(L, B, 8, 1, 128), new_rows=0, max_len=90, mass_stride=101)


@pytest.mark.parametrize("new_rows,T", [(1, 1), (3, 3), (4, 2)])
def test_new_rows_and_one_length_for_all(new_rows, T):
    c = Cache(1, 2, 2, 128, 16, 8, "bf16", len_uniform=70)
    _check(c, _q(1, 2, 4, T, 128), T, new_rows)


@pytest.mark.parametrize("scale,spread", [(0.0, 12.0), (3.0, 1.0), (1e-4, 1.0)])
def test_sharp_and_flat_scores(scale, spread):
    c = Cache(1, 2, 2, 128, 16, 40, "bf16", lens=[640, 333], scale=spread)
    _check(c, _q(1, 2, 8, 1, 128, scale=spread), scale=scale)


@pytest.mark.parametrize("form", ["e4m3", "int8"])
def test_scales_far_apart(form):
    c = Cache(1, 1, 1, 128, 16, 20, form, lens=[300])
    for name, span in (("k_scale", 0.5), ("v_scale", 12.0)):  # values over ten orders of magnitude
        s = c.dev[name]
        s *= torch.exp(span * torch.randn(s.shape, generator=torch.Generator().manual_seed(1)).to(DEV))
    _check(c, _q(1, 1, 4, 1, 128))
    c.dev["v_scale"] *= 1e-30
    _check(c, _q(1, 1, 4, 1, 128))


@pytest.mark.parametrize("layout,d_rot,G,T", [(0, 128, 4, 1), (1, 64, 4, 1), (0, 40, 3, 4), (1, 128, 16, 2)])
@pytest.mark.parametrize("given", [False, True])
def test_rotated_queries(layout, d_rot, G, T, given):
    lens = [9, 200]
    c = Cache(1, 2, 2, 128, 16, 14, "bf16", lens=lens)
    pos = torch.randint(0, 100000, (2, T), generator=torch.Generator().manual_seed(1), dtype=torch.int32) if given else None
    rot, keep = rotary(d_rot, layout, magnitude=1.1, positions=pos.to(DEV) if given else None)
    _check(c, _q(1, 2, 2 * G, T, 128), T, rot=rot, ref_rot=(frequencies(d_rot), d_rot, layout == 1, 1.1, False, pos))


def test_strided_queries_and_outputs():
    L, B, H, T, d = 2, 3, 6, 2, 64
    c = Cache(L, B, 2, d, 16, 5, "bf16", lens=[70, 3, 41])
    big = _q(L, B, H, T, d).to(DEV)
    x = torch.zeros((L, B, T, H + 4, d + 64), dtype=torch.bfloat16, device=DEV)
    x[:, :, :, 2:2 + H, 64:] = big.transpose(2, 3)
    out = torch.full((L + 1, B, T, H, d + 8), 7.0, dtype=torch.bfloat16, device=DEV)
    view = out[..., :d].transpose(2, 3)
    got = run_attend(c, x[:, :, :, 2:2 + H, 64:].transpose(2, 3), T, out=view)
    want = run_attend(c, big, T)
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    assert (out[..., d:] == 7.0).all()


@pytest.mark.parametrize("form", ["bf16", "e4m3"])
@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
def test_what_is_not_seen_has_no_influence(form, bad):
    lens, T = [0, 5, 16, 83], 4
    q = _q(1, 4, 8, T, 128)

    def fill(c, value):
        for name in ("k", "v"):
            for b, n in enumerate(lens):  # behind the last row of every sequence, and the pages that nobody owns
                for r in range(n, c.wide * c.page):
                    at, off = int(c.page_ids(b)[r // c.page]), r % c.page
                    if form == "bf16":
                        c.dev[name][:, at, :, off] = value
                    else:
                        c.dev[name + "_scale"][:, at, :, off] = value
        return c

    plain = run_attend(fill(Cache(1, 4, 2, 128, 16, 8, form, lens=lens), 0.0), q.to(DEV), T)
    dirty = run_attend(fill(Cache(1, 4, 2, 128, 16, 8, form, lens=lens), bad), q.to(DEV), T)
    for a, b in zip(plain, dirty):
        assert torch.equal(a, b)
    # rows that a later token sees and an earlier one does not
    c = Cache(1, 4, 2, 128, 16, 8, form, lens=lens)
    clean = run_attend(c, q.to(DEV), T)
    for b, n in ((1, 5), (3, 83)):
        at, off = int(c.page_ids(b)[(n - 2) // 16]), (n - 2) % 16
        if form == "bf16":
            c.dev["v"][:, at, :, off] = bad
        else:
            c.dev["v_scale"][:, at, :, off] = bad
    got = run_attend(c, q.to(DEV), T)
    for b in (1, 3):
        assert torch.equal(got[0][:, b, :, :T - 2], clean[0][:, b, :, :T - 2])  # they do not see row n - 2
        assert not torch.isfinite(got[0][:, b, :, T - 2:]).all()  # those that see it are told
    assert torch.equal(got[1], clean[1]) and torch.equal(got[2], clean[2])  # the scores do not depend on values


def test_nan_in_a_seen_key_is_told():
    c = Cache(1, 1, 1, 128, 16, 2, "bf16", lens=[20])
    c.dev["k"][0, int(c.page_ids(0)[0]), 0, 3, 5] = math.nan
    got = run_attend(c, _q(1, 1, 2, 1, 128).to(DEV), 1)
    assert got[0].isnan().all() and got[1].isnan().all()


def test_unseen_pages_of_the_table_are_not_read():
    c = Cache(1, 2, 1, 128, 16, 4, "bf16", lens=[20, 33])
    want = run_attend(c, _q(1, 2, 4, 1, 128).to(DEV), 1)
    c.d_table[0, 2:] = -1
    c.d_table[1, 3:] = 2 ** 31 - 1
    got = run_attend(c, _q(1, 2, 4, 1, 128).to(DEV), 1)
    assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_what_is_outside_is_cut_and_reported():
    c = Cache(1, 3, 1, 128, 16, 4, "bf16", lens=[64, 70, 40])
    q = _q(1, 3, 4, 1, 128).to(DEV)
    with Ctx(1 << 22) as h:
        got = run_attend(c, q, 1, ctx=h)
        assert ta.ta_ctx_poll(h) == ta.TA_ERR_DEVICE_BOUNDS  # 70 rows do not fit 4 pages
        c.lens, c.d_lens = [64, 64, 40], torch.tensor([64, 64, 40], dtype=torch.int32, device=DEV)
        want = run_attend(c, q, 1, ctx=h)
        assert ta.ta_ctx_poll(h) == ta.TA_OK
        assert all(torch.equal(a, b) for a, b in zip(got, want))
        run_attend(c, q, 1, max_len=63, ctx=h)
        assert ta.ta_ctx_poll(h) == ta.TA_ERR_DEVICE_BOUNDS
        c.d_table[2, 1] = c.pages  # rows 16..31 lie nowhere
        got = run_attend(c, q, 1, ctx=h)
        assert ta.ta_ctx_poll(h) == ta.TA_ERR_DEVICE_BOUNDS
    keep = [r for r in range(40) if not 16 <= r < 32]
    k, v = (c.rows(n, 0, 2, 0, 16).clone() for n in ("k", "v"))
    last = int(c.table[2, 2])
    k, v = (torch.cat((x, c.dev[n][0, last, 0, :8].cpu().double())) for n, x in (("k", k), ("v", v)))
    s = q[0, 2, :, 0].cpu().double() @ k.T / math.sqrt(128)
    assert ((s.softmax(-1) @ v - got[0][0, 2, :, 0]).abs() <= 2.0 ** -7 * 4).all()
    assert (got[2][0, 2, 0, 16:32] == 0).all() and len(keep) == 24


def test_another_stream_repeats_and_a_shared_context():
    c = Cache(1, 2, 2, 128, 16, 300, "bf16", lens=[4700, 33])
    q = _q(1, 2, 8, 1, 128).to(DEV)
    with Ctx(1 << 26) as h:
        first = run_attend(c, q, 1, ctx=h)
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            again = run_attend(c, q, 1, ctx=h)
        for _ in range(5):
            more = run_attend(c, q, 1, ctx=h)
            assert all(torch.equal(a, b) for a, b in zip(first, more))
        assert ta.ta_ctx_poll(h) == ta.TA_OK
    assert all(torch.equal(a, b) for a, b in zip(first, again))


def test_in_a_graph():
    c = Cache(1, 2, 2, 128, 16, 60, "e4m3", lens=[900, 33])
    q = _q(1, 2, 8, 1, 128).to(DEV)
    want = run_attend(c, q, 1)
    s = c.struct()
    out, lse, mass = torch.zeros_like(q), torch.zeros((1, 2, 8, 1), device=DEV), torch.zeros((1, 2, 2, 960), device=DEV)
    with Ctx(1 << 24) as h:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            ta.ta_attend(h, s, 8, 1, 0, 960, True, 0.0, None, ta.view(q), ta.view(out), lse, mass, 960,
                         torch.cuda.current_stream().cuda_stream)
        for _ in range(3):
            out.zero_()
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(out.cpu().double(), want[0]) and torch.equal(mass.cpu().double(), want[2])
        assert ta.ta_ctx_poll(h) == ta.TA_OK
        del graph


def test_refusals():
    c = Cache(1, 2, 2, 128, 16, 2, "int8", lens=[3, 4])
    x = torch.zeros((1, 2, 4, 1, 128), dtype=torch.bfloat16, device=DEV)
    v, mass = ta.view(x), torch.zeros((1, 2, 2, 32), device=DEV)
    with Ctx(1 << 22) as h:
        def status(s=None, Hq=4, T=1, new=0, most=32, scale=0.0, rot=None, q=v, out=v, m=None, stride=0, ctx=h):
            with pytest.raises(ta.TAError) as e:
                ta.ta_attend(ctx, s or c.struct(), Hq, T, new, most, True, scale, rot, q, out, None, m, stride)
            return e.value.status
        for s, want in _bad_caches():
            if want == ta.TA_ERR_INVALID_ARG and (s.batch == 3 or s.n_layers == 2):
                continue  # there the batch of the call says otherwise
            assert status(s) == want
        assert status(Hq=3) == ta.TA_ERR_INVALID_ARG and status(Hq=0) == ta.TA_ERR_INVALID_ARG
        assert status(T=0) == ta.TA_ERR_INVALID_ARG and status(T=65) == ta.TA_ERR_UNSUPPORTED
        assert status(Hq=2 * 257) == ta.TA_ERR_UNSUPPORTED
        assert status(new=-1) == ta.TA_ERR_INVALID_ARG and status(most=-1) == ta.TA_ERR_INVALID_ARG
        assert status(most=(1 << 20) + 1) == ta.TA_ERR_UNSUPPORTED
        assert status(scale=-1.0) == ta.TA_ERR_INVALID_ARG and status(scale=math.nan) == ta.TA_ERR_INVALID_ARG
        assert status(rot=ta.make_rotary(None, 128)) == ta.TA_ERR_INVALID_ARG
        assert status(q=ta.view(None)) == ta.TA_ERR_INVALID_ARG
        assert status(out=ta.ta_bf16_view(x.data_ptr() + 2, 1024, 512, 128, 128)) == ta.TA_ERR_ALIGNMENT
        assert status(m=mass, stride=31) == ta.TA_ERR_INVALID_ARG
        assert status(ctx=None) == ta.TA_ERR_INVALID_ARG
        assert ta.ta_ctx_poll(h) == ta.TA_OK
    with Ctx(0) as h:
        need = ta.ta_attend_scratch_bytes(c.struct(), 4, 1, 32, True)
        assert need > 0 and status(m=mass, stride=32, ctx=h) == ta.TA_ERR_SCRATCH_TOO_SMALL

"""Writing a cache in its format and reading it back: codes bit for bit as documented, values against 64 bits, addressing."""
import math

import pytest
import torch

import paper_2604_11288_b200 as ta
from decode_testlib import DEV, FULL, TYPES, U, Cache, Ctx, codes, frequencies, rotary, rotated, within

pytestmark = pytest.mark.gpu
STREAM = (lambda: torch.cuda.current_stream().cuda_stream)


def _append(c, k, v, batch, rot=None, rows=None, ragged=False, ok=True):
    with Ctx() as h:
        ta.ta_cache_append(h, c.struct(), batch, rot, ta.view(k, ragged), ta.view(v, ragged), rows, STREAM())
        assert ta.ta_ctx_poll(h) == (ta.TA_OK if ok else ta.TA_ERR_DEVICE_BOUNDS)


def _read(c, shape, batch, rows=None, ragged=False, ok=True):
    ko, vo = (torch.full(shape, 7.0, dtype=torch.bfloat16, device=DEV) for _ in range(2))
    with Ctx() as h:
        ta.ta_cache_read(h, c.struct(), batch, rows, ta.view(ko, ragged), ta.view(vo, ragged), STREAM())
        assert ta.ta_ctx_poll(h) == (ta.TA_OK if ok else ta.TA_ERR_DEVICE_BOUNDS)
    return ko, vo


def _raw(t):
    return (t.view(torch.int8) if t.element_size() == 1 else t.view(torch.int16)).cpu()


def _where(c, b, row):
    return int(c.page_ids(b)[row // c.page]), row % c.page


@pytest.mark.parametrize("form", ["bf16", "e4m3", "int8"])
@pytest.mark.parametrize("order", ["heads", "rows"])
@pytest.mark.parametrize("d,page,kv", [(128, 16, 2), (64, 1, 3), (128, 13, 1), (64, 64, 8)])
def test_ragged_prompt_codes_and_back(form, order, d, page, kv):
    g = torch.Generator().manual_seed(page)
    lens, held = [5, 0, 33, 1], [0, 3, 14, 7]
    L, B, total = 2, len(lens), sum(lens)
    c = Cache(L, B, kv, d, page, -(-48 // page), form, order, lens=held, seed=1)
    before = {n: _raw(c.dev[n]).clone() for n in ("k", "v")}
    x = {n: (torch.randn((L, total, kv, d), generator=g) * torch.exp(3 * torch.randn((L, total, kv, 1), generator=g))).to(torch.bfloat16)
         for n in ("k", "v")}
    x["k"][0, 0, 0], x["v"][1, 2, 0] = 0.0, 1e-38  # a row of zeros, one below the smallest largest value
    x["k"][1, 3, 0, 5], x["v"][0, 4, 0, 1] = math.nan, math.inf
    dk, dv = (x[n].to(DEV).transpose(1, 2) for n in ("k", "v"))
    cu = torch.tensor([sum(lens[:i]) for i in range(B + 1)], dtype=torch.int32, device=DEV)
    batch = ta.make_batch(L, B, 0, max(lens), total, cu)
    _append(c, dk, dv, batch, ragged=True)
    touched = {n: torch.zeros(before[n].shape[:4], dtype=torch.bool) for n in ("k", "v")}
    rows = torch.cat([torch.arange(n) + h for n, h in zip(lens, held)])
    seq = torch.repeat_interleave(torch.arange(B), torch.tensor(lens))
    rows_all = rows.int().expand(L, kv, total).contiguous().to(DEV)
    back = dict(zip(("k", "v"), _read(c, (L, kv, total, d), batch, rows_all, ragged=True)))
    for n in ("k", "v"):
        code, scale = codes(x[n].float(), form) if form != "bf16" else (x[n], None)
        for i in range(total):
            at, off = _where(c, int(seq[i]), int(rows[i]))
            touched[n][:, at, :, off] = True
            assert torch.equal(_raw(c.dev[n])[:, at, :, off], _raw(code)[:, i]), (n, i)
            if scale is not None:
                s = c.dev[n + "_scale"].cpu()[:, at, :, off]
                assert torch.equal(s.nan_to_num(-1.0), scale[:, i].nan_to_num(-1.0))
        untouched = ~touched[n]
        assert torch.equal(_raw(c.dev[n])[untouched], before[n][untouched])
        got = back[n].cpu().transpose(1, 2)
        want = code if scale is None else (code.float() * scale.unsqueeze(-1)).to(torch.bfloat16)
        assert torch.equal(got.isnan(), want.isnan()) and torch.equal(got.nan_to_num(0.0), want.nan_to_num(0.0))
        if scale is not None:  # and near what was written: half a step of the format, then bf16
            fine = torch.isfinite(x[n].float()).all(-1, keepdim=True).expand(x[n].shape)
            y, top = x[n].double(), x[n].double().abs().amax(-1, keepdim=True)
            step = top / 254 if form == "int8" else torch.maximum(y.abs() * 2.0 ** -4, top / 448 * 2.0 ** -10)
            lost = 1e-30  # what is below 2^-100 / 448 is not told from zero
            within(got.double()[fine], y[fine], ((step + U * y.abs()) * 1.01 + lost)[fine], n)


@pytest.mark.parametrize("form", ["bf16", "e4m3", "int8"])
@pytest.mark.parametrize("d,d_rot,layout", [(128, 128, 0), (128, 64, 1), (64, 24, 0), (64, 64, 1)])
def test_rotated_on_the_way(form, d, d_rot, layout):
    g = torch.Generator().manual_seed(7)
    L, B, kv, n = 1, 3, 2, 9
    held = [0, 100, 31]
    c = Cache(L, B, kv, d, 16, 8, form, lens=held)
    k, v = (torch.randn((L, B, kv, n, d), generator=g).to(torch.bfloat16).to(DEV) for _ in range(2))
    rot, keep = rotary(d_rot, layout)
    _append(c, k, v, ta.make_batch(L, B, n, n, B * n), rot)
    f = frequencies(d_rot)
    for b in range(B):
        for h in range(kv):
            x = k[0, b, h].cpu().double()
            y = rotated(x, torch.arange(n) + held[b], f, d_rot, layout == 1)
            top = y.abs().amax(-1, keepdim=True)
            step = {"bf16": U * y.abs(), "int8": top / 254, "e4m3": torch.maximum(y.abs() * 2.0 ** -4, top / 448 * 2.0 ** -10)}[form]
            tol = step * 1.01 + 2.0 ** -19 * x.abs().amax(-1, keepdim=True)
            within(c.rows("k", 0, b, h, held[b] + n)[held[b]:], y, tol, "k")
            code, scale = codes(v[0, b, h].cpu().float(), form)
            want = code.double() if scale is None else code.float().double() * scale.double().unsqueeze(-1)
            assert torch.equal(c.rows("v", 0, b, h, held[b] + n)[held[b]:], want)
    # given positions in place of the rows
    pos = torch.randint(0, 100000, (B * n,), generator=g, dtype=torch.int32)
    rot, keep = rotary(d_rot, layout, positions=pos.to(DEV))
    _append(c, k, v, ta.make_batch(L, B, n, n, B * n), rot)
    for b in range(B):
        x = k[0, b, 0].cpu().double()
        y = rotated(x, pos.view(B, n)[b], f, d_rot, layout == 1)
        top = y.abs().amax(-1, keepdim=True)
        step = {"bf16": U * y.abs(), "int8": top / 254, "e4m3": torch.maximum(y.abs() * 2.0 ** -4, top / 448 * 2.0 ** -10)}[form]
        within(c.rows("k", 0, b, 0, held[b] + n)[held[b]:], y, step * 1.01 + 2.0 ** -19 * x.abs().amax(-1, keepdim=True), "k")


@pytest.mark.parametrize("form", ["bf16", "e4m3", "int8"])
def test_rows_by_index_dense_and_per_unit(form):
    g = torch.Generator().manual_seed(9)
    L, B, kv, d, K = 2, 2, 3, 128, 37
    c = Cache(L, B, kv, d, K + 1, 1, form, dense=True, seed=4)
    k, v = (torch.randn((L, B, 1, kv, d), generator=g).to(torch.bfloat16).to(DEV).transpose(2, 3) for _ in range(2))
    rows = torch.randint(0, K + 1, (L, B, kv, 1), generator=g, dtype=torch.int32)
    rows[0, 0, 0, 0] = -1
    old = c.rows("k", 0, 0, 0, K + 1)
    _append(c, k, v, ta.make_batch(L, B, 1, 1, B), rows=rows.to(DEV))
    assert torch.equal(c.rows("k", 0, 0, 0, K + 1), old)  # not written
    idx = torch.full((L, B, kv, 5), -1, dtype=torch.int32)
    idx[..., 1] = rows[..., 0].clamp_min(0)
    idx[..., 3] = K
    ko, vo = _read(c, (L, B, kv, 5, d), ta.make_batch(L, B, 5, 5, B * 5), idx.to(DEV))
    for l in range(L):
        for b in range(B):
            for h in range(kv):
                for name, out, x in (("k", ko, k), ("v", vo, v)):
                    held = c.rows(name, l, b, h, K + 1)
                    want = torch.zeros(5, d, dtype=torch.float64)
                    want[1], want[3] = held[int(idx[l, b, h, 1])], held[K]
                    assert torch.equal(out[l, b, h].cpu(), want.float().to(torch.bfloat16))
                    if rows[l, b, h, 0] >= 0 and form == "bf16":
                        assert torch.equal(out[l, b, h, 1], x[l, b, h, 0])


def test_rows_outside_are_reported_and_skipped():
    c = Cache(1, 2, 1, 128, 16, 2, "int8", lens=[30, 31])
    c.d_table[1, 1] = c.pages  # no such page
    c.d_table[0, 1] = -1
    before = _raw(c.dev["k"]).clone()
    k = torch.ones((1, 2, 1, 1, 128), dtype=torch.bfloat16, device=DEV)
    one = ta.make_batch(1, 2, 1, 1, 2)
    _append(c, k, k, one, ok=False)
    rows = torch.tensor([32, 2 ** 31 - 1], dtype=torch.int32, device=DEV).view(1, 2, 1, 1)
    _append(c, k, k, one, rows=rows, ok=False)
    assert torch.equal(_raw(c.dev["k"]), before)
    ko, vo = _read(c, (1, 2, 1, 1, 128), one, rows, ok=False)
    assert (ko == 0).all() and (vo == 0).all()
    ko, vo = _read(c, (1, 2, 1, 1, 128), one, torch.full_like(rows, 31), ok=False)
    assert (ko == 0).all()


@pytest.mark.parametrize("form", ["bf16", "e4m3"])
def test_offsets_beyond_32_bits(form):
    wide = 3 << 30  # bytes between pages
    size = 2 if form == "bf16" else 1
    kv, page, d = 2, 4, 128
    pools = [torch.zeros(2 * wide + (1 << 16), dtype=torch.uint8, device=DEV).view(TYPES[form]) for _ in range(2)]
    shape, stride = (1, 3, kv, page, d), (0, wide // size, page * d, d, 1)
    k, v = (p.as_strided(shape, stride) for p in pools)
    ks, vs = (torch.zeros((1, 3, kv, page), device=DEV) if size == 1 else None for _ in range(2))
    table = torch.tensor([[2, 0, 1]], dtype=torch.int32, device=DEV)
    c = ta.make_cache(k, v, ks, vs, table=table, len_uniform=0)
    g = torch.Generator().manual_seed(2)
    x, y = (torch.randn((1, 1, kv, 12, d), generator=g).to(torch.bfloat16).to(DEV) for _ in range(2))
    batch = ta.make_batch(1, 1, 12, 12, 12)
    ko, vo = torch.empty_like(x), torch.empty_like(x)
    c.len_uniform = 0
    q, out = (torch.randn((1, 1, 4, 1, d), generator=g).to(torch.bfloat16).to(DEV) for _ in range(2))
    with Ctx(1 << 22) as h:
        ta.ta_cache_append(h, c, batch, None, ta.view(x), ta.view(y), None, STREAM())
        ta.ta_cache_read(h, c, batch, None, ta.view(ko), ta.view(vo), STREAM())
        ta.ta_attend(h, c, 4, 1, 12, 12, True, 0.0, None, ta.view(q), ta.view(out), None, None, 0, STREAM())
        assert ta.ta_ctx_poll(h) == ta.TA_OK
    for a, b in ((x, ko), (y, vo)):
        code, scale = codes(a.cpu().float(), form)
        want = code if scale is None else (code.float() * scale.unsqueeze(-1)).to(torch.bfloat16)
        assert torch.equal(b.cpu(), want)
    s = torch.einsum("lbgqd,lbgnd->lbgqn", q.cpu().double().view(1, 1, kv, 2, d), ko.cpu().double()) / math.sqrt(d)
    want = torch.einsum("lbgqn,lbgnd->lbgqd", s.softmax(-1), vo.cpu().double())
    # read back values were rounded to bf16 once more than the attention's: 2^-8 of scores below 8 and of values
    assert ((out.cpu().double().view(want.shape) - want).abs() <= 0.08).all()
    del pools


def test_another_stream_and_repeats():
    c = Cache(1, 4, 2, 128, 16, 40, "e4m3", lens=[0] * 4)
    g = torch.Generator().manual_seed(3)
    k, v = (torch.randn((1, 4, 2, 600, 128), generator=g).to(torch.bfloat16).to(DEV) for _ in range(2))
    batch = ta.make_batch(1, 4, 600, 600, 2400)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    got = []
    with Ctx() as h:
        for _ in range(2):
            ko, vo = torch.empty_like(k), torch.empty_like(v)
            side.wait_stream(torch.cuda.current_stream())
            ta.ta_cache_append(h, c.struct(), batch, None, ta.view(k), ta.view(v), None, side.cuda_stream)
            ta.ta_cache_read(h, c.struct(), batch, None, ta.view(ko), ta.view(vo), side.cuda_stream)
            side.synchronize()
            got.append((ko.cpu(), vo.cpu()))
        assert ta.ta_ctx_poll(h) == ta.TA_OK
    assert torch.equal(got[0][0], got[1][0]) and torch.equal(got[0][1], got[1][1])
    code, scale = codes(k.cpu().float(), "e4m3")
    assert torch.equal(got[0][0], (code.float() * scale.unsqueeze(-1)).to(torch.bfloat16))


def _bad_caches():
    def change(**kw):
        s = Cache(1, 2, 2, 128, 16, 2, kw.pop("form", "int8")).struct()
        for n, x in kw.items():
            setattr(s, n, x)
        return s
    yield change(k=None), ta.TA_ERR_INVALID_ARG
    yield change(k_scale=None), ta.TA_ERR_INVALID_ARG
    yield change(format=3), ta.TA_ERR_INVALID_ARG
    yield change(page=0), ta.TA_ERR_INVALID_ARG
    yield change(n_pages=0), ta.TA_ERR_INVALID_ARG
    yield change(pages_per_seq=0), ta.TA_ERR_INVALID_ARG
    yield change(batch=3), ta.TA_ERR_INVALID_ARG
    yield change(n_layers=2), ta.TA_ERR_INVALID_ARG
    yield change(d=96), ta.TA_ERR_UNSUPPORTED
    yield change(stride_h=-16), ta.TA_ERR_INVALID_ARG
    yield change(stride_h=8), ta.TA_ERR_ALIGNMENT
    yield change(stride_r=64), ta.TA_ERR_INVALID_ARG
    yield change(scale_stride_r=-1), ta.TA_ERR_INVALID_ARG
    yield change(lens=None, len_uniform=-1), ta.TA_ERR_INVALID_ARG
    yield change(form="bf16", stride_l=4), ta.TA_ERR_ALIGNMENT


def test_refusals():
    x = torch.zeros((1, 2, 2, 1, 128), dtype=torch.bfloat16, device=DEV)
    batch, view = ta.make_batch(1, 2, 1, 1, 2), ta.view(x)
    good = Cache(1, 2, 2, 128, 16, 2, "int8", lens=[0, 0])
    with Ctx() as h:
        for s, status in _bad_caches():
            for call in (lambda: ta.ta_cache_append(h, s, batch, None, view, view), lambda: ta.ta_cache_read(h, s, batch, None, view, view)):
                with pytest.raises(ta.TAError) as e:
                    call()
                assert e.value.status == status
        odd = ta.ta_bf16_view(x.data_ptr() + 8, 512, 256, 128, 128)
        for s, status in ((odd, ta.TA_ERR_ALIGNMENT), (ta.view(None), ta.TA_ERR_INVALID_ARG)):
            for call in (lambda: ta.ta_cache_append(h, good.struct(), batch, None, view, s),
                         lambda: ta.ta_cache_read(h, good.struct(), batch, None, s, view)):
                with pytest.raises(ta.TAError) as e:
                    call()
                assert e.value.status == status
        with pytest.raises(ta.TAError):
            ta.ta_cache_append(h, good.struct(), batch, ta.make_rotary(None, 128), view, view)
        assert ta.ta_ctx_poll(h) == ta.TA_OK
    assert FULL["int8"] == 127.0

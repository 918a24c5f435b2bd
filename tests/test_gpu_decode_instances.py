"""The kernel variants of the decode loop's operators that a call's size picks, each on its side of the threshold: blocks of two warps for
many short units, more units than counters, cuts of more units than run at once, 32 rows a block of the cache kernels, batches whose
lengths are not kept in shared memory, several tokens a thread of the rotation."""
import pytest
import torch

import paper_2604_11288_b200 as ta
from decode_batched import attend, held_rows, rotated
from decode_testlib import DEV, U, Cache, Ctx, codes, frequencies, rotary, run_attend, within

pytestmark = pytest.mark.gpu
STREAM = (lambda: torch.cuda.current_stream().cuda_stream)


def _randn(*shape, seed=0, dtype=torch.bfloat16):
    g = torch.Generator(device=DEV).manual_seed(seed)
    return torch.randn(shape, generator=g, device=DEV).to(dtype)


def _check_attend(c, q, T, lens, causal=True, rot=None, ref_rot=None, **kw):
    got = run_attend(c, q, T, causal=causal, rot=rot, **kw)
    out, lse, mass, tol, lse_tol, mass_tol = attend(c, q, T, lens, causal, ref_rot)
    within(got[0], out, tol, "out")
    within(got[1], lse, lse_tol, "lse")
    if got[2] is not None:
        n = mass.shape[-1]
        within(got[2][..., :n], mass, mass_tol, "mass")
        assert (got[2][..., n:] == 0).all()


# ---- attention -------------------------------------------------------------------------------------------------------------------


@pytest.mark.parametrize("form", ["bf16", "e4m3", "int8"])
@pytest.mark.parametrize("d,G,T", [(128, 4, 1), (64, 1, 8), (128, 2, 3), (64, 7, 1)])
@pytest.mark.parametrize("lengths", ["per unit", "per sequence", "one"])
def test_many_short_units(form, d, G, T, lengths):
    """1800 units of up to 8 query rows: blocks of two warps."""
    L, B, kv, most = 3, 75, 8, 70
    g = torch.Generator().manual_seed(d + G)
    if lengths == "per unit":
        lens = torch.randint(0, most + 1, (L, B, kv), generator=g)
        own = lens.tolist()
    elif lengths == "per sequence":
        own = torch.randint(0, most + 1, (B,), generator=g).tolist()
        lens = torch.tensor(own).view(1, B, 1).expand(L, B, kv)
    else:
        own, lens = None, torch.full((L, B, kv), most)
    c = Cache(L, B, kv, d, 13, 6, form, "rows", lens=own, len_uniform=most, seed=G)
    _check_attend(c, _randn(L, B, T, kv * G, d).transpose(2, 3), T, lens, max_len=most, mass_stride=most + 3)


@pytest.mark.parametrize("form", ["bf16", "int8"])
@pytest.mark.parametrize("layout,d_rot,given", [(0, 128, False), (1, 64, True), (0, 40, False)])
def test_many_short_units_with_rotated_queries(form, layout, d_rot, given):
    L, B, kv, G, T, most = 2, 120, 8, 2, 2, 65
    g = torch.Generator().manual_seed(d_rot)
    lens = torch.randint(0, most + 1, (B,), generator=g)
    pos = torch.randint(0, 100000, (B, T), generator=g, dtype=torch.int32) if given else None
    rot, keep = rotary(d_rot, layout, magnitude=0.9, positions=pos.to(DEV) if given else None)
    c = Cache(L, B, kv, 128, 16, 5, form, lens=lens.tolist(), seed=2)
    _check_attend(c, _randn(L, B, kv * G, T, 128), T, lens.view(1, B, 1).expand(L, B, kv), rot=rot,
                  ref_rot=(frequencies(d_rot), d_rot, layout == 1, 0.9, pos), max_len=most, mass_stride=most)


@pytest.mark.parametrize("form", ["bf16", "e4m3"])
def test_a_step_of_257_rows_in_every_unit(form):
    """Two-warp blocks of many tiles, the last one partly filled."""
    L, B, kv = 5, 64, 8
    c = Cache(L, B, kv, 128, 257, 1, form, dense=True, len_uniform=257, seed=3)
    _check_attend(c, _randn(L, B, 32, 1, 128), 1, torch.full((L, B, kv), 257))


@pytest.mark.parametrize("form,G,T,B", [("bf16", 1, 1, 2051), ("int8", 4, 2, 2051), ("e4m3", 16, 1, 2051), ("bf16", 8, 8, 1030)])
def test_more_row_blocks_than_counters(form, G, T, B):
    """Over 16384 of them: one piece each, whatever the length."""
    kv, n = 8, 150
    lens = torch.randint(0, n + 1, (B,), generator=torch.Generator().manual_seed(B))
    c = Cache(1, B, kv, 64, 75, 2, form, lens=lens.tolist(), seed=5)
    _check_attend(c, _randn(1, B, kv * G, T, 64), T, lens.view(1, B, 1).expand(1, B, kv), with_mass=False)


@pytest.mark.parametrize("form", ["bf16", "e4m3", "int8"])
@pytest.mark.parametrize("G,T", [(4, 1), (4, 4), (4, 8)])
def test_more_units_than_run_at_once_in_pieces(form, G, T):
    """512 units: cut all the same, for lengths that differ."""
    B, kv, n = 64, 8, 1100
    lens = torch.randint(0, n + 1, (B,), generator=torch.Generator().manual_seed(T))
    lens[3], lens[4] = 0, n
    c = Cache(1, B, kv, 64, 50, 22, form, lens=lens.tolist(), seed=6)
    _check_attend(c, _randn(1, B, kv * G, T, 64), T, lens.view(1, B, 1).expand(1, B, kv), with_mass=T == 1)


@pytest.mark.parametrize("form", ["bf16", "int8"])
@pytest.mark.parametrize("B", [2, 222, 377, 444, 445])
def test_lengths_added_up_on_the_device(form, B):
    """Sequences of one unit each, up to 377 of them cut by the sum of their lengths."""
    lens = torch.randint(0, 401, (B,), generator=torch.Generator().manual_seed(B))
    lens[1], lens[0] = 400, 0
    c = Cache(1, B, 1, 128, 16, 25, form, lens=lens.tolist(), seed=7)
    _check_attend(c, _randn(1, B, 4, 1, 128), 1, lens.view(1, B, 1))


# ---- the cache -------------------------------------------------------------------------------------------------------------------


def _steps(y, form):
    """What a format's rounding may cost: half a step, as in decode_testlib's tolerances."""
    top = y.abs().amax(-1, keepdim=True)
    return {"bf16": U * y.abs(), "int8": (top / 254).expand(y.shape),
            "e4m3": torch.maximum(y.abs() * 2.0 ** -4, top / 448 * 2.0 ** -10)}[form]


@pytest.mark.parametrize("form", ["bf16", "e4m3", "int8"])
@pytest.mark.parametrize("d,d_rot,layout,kv", [(128, 128, 0, 5), (128, 64, 1, 8), (64, 64, 0, 3), (64, 24, 0, 1), (128, 104, 0, 2), (64, 40, 1, 33)])
@pytest.mark.parametrize("ragged,given", [(True, False), (True, True), (False, False)])
def test_rotated_on_the_way_32_rows_a_block(form, d, d_rot, layout, kv, ragged, given):
    g = torch.Generator().manual_seed(d_rot + kv)
    L, B = 2, 7
    each = -(-5000 // (L * B * kv))
    lens = torch.randint(0, 2 * each, (B,), generator=g) if ragged else torch.full((B,), each)
    if ragged:
        lens[2], lens[5] = 0, 3 * each
    total, held = int(lens.sum()), torch.randint(0, 90, (B,), generator=g)
    if L * total * kv <= 4736:
        lens[0] += 5000 // (L * kv)
        total = int(lens.sum())
    assert L * total * kv > 4736
    most = int((lens + held).max())
    c = Cache(L, B, kv, d, 16, -(-most // 16), form, "rows", lens=held.tolist(), seed=1)
    k, v = (_randn(L, total, kv, d, seed=s) for s in (1, 2))
    pos = torch.randint(0, 100000, (total,), generator=g, dtype=torch.int32) if given else None
    rot, keep = rotary(d_rot, layout, positions=None if pos is None else pos.to(DEV))
    seq = torch.repeat_interleave(torch.arange(B), lens)
    index = torch.cat([torch.arange(int(n)) for n in lens])
    rows = index + held[seq]
    if ragged:
        cu = torch.tensor([0] + lens.cumsum(0).tolist(), dtype=torch.int32, device=DEV)
        batch = ta.make_batch(L, B, 0, int(lens.max()), total, cu)
        kk, vv = k.transpose(1, 2), v.transpose(1, 2)
    else:
        batch = ta.make_batch(L, B, each, each, total)
        kk, vv = (x.view(L, B, each, kv, d).transpose(2, 3) for x in (k, v))
    with Ctx() as h:
        ta.ta_cache_append(h, c.struct(), batch, rot, ta.view(kk, ragged), ta.view(vv, ragged), None, STREAM())
        assert ta.ta_ctx_poll(h) == ta.TA_OK
    x = k.double()
    want = rotated(x, (rows if pos is None else pos).to(DEV).view(1, total, 1), frequencies(d_rot), d_rot, layout == 1)
    at = (lambda name: held_rows(c, name, most).transpose(1, 2)[:, :, seq.to(DEV), rows.to(DEV)].transpose(1, 2))
    within(at("k"), want, _steps(want, form) * 1.01 + 2.0 ** -19 * x.abs().amax(-1, keepdim=True), "k")
    got = at("v")
    code, scale = codes(v.cpu().float(), form)
    want = code.double() if scale is None else code.float().double() * scale.double().unsqueeze(-1)
    assert torch.equal(got.cpu(), want)


@pytest.mark.parametrize("form", ["bf16", "e4m3", "int8"])
@pytest.mark.parametrize("d,kv,B,L", [(128, 3, 300, 2), (64, 8, 257, 3), (64, 1, 256, 20), (128, 2, 300, 1)])
@pytest.mark.parametrize("ragged", [True, False])
def test_written_and_read_back_in_large_batches(form, d, kv, B, L, ragged):
    """Batches around 256 sequences, above and below 4736 rows; codes bit for bit, and the rest of the pool untouched."""
    g = torch.Generator().manual_seed(B + kv)
    each = 4
    lens = torch.randint(0, 2 * each, (B,), generator=g) if ragged else torch.full((B,), each)
    held, total = torch.randint(0, 30, (B,), generator=g), int(lens.sum())
    c = Cache(L, B, kv, d, 7, 6, form, lens=held.tolist(), seed=2)
    k, v = (_randn(L, total, kv, d, seed=s) for s in (3, 4))
    k *= torch.exp(2 * _randn(L, total, kv, 1, seed=5))
    before = [held_rows(c, n, 42) for n in ("k", "v")]
    seq, index = torch.repeat_interleave(torch.arange(B), lens), torch.cat([torch.arange(int(n)) for n in lens])
    rows = index + held[seq]
    if ragged:
        cu = torch.tensor([0] + lens.cumsum(0).tolist(), dtype=torch.int32, device=DEV)
        batch = ta.make_batch(L, B, 0, int(lens.max()), total, cu)
        kk, vv = k.transpose(1, 2), v.transpose(1, 2)
        index_of = rows.int().expand(L, kv, total).contiguous().to(DEV)
        shape = (L, kv, total, d)
    else:
        batch = ta.make_batch(L, B, each, each, total)
        kk, vv = (x.view(L, B, each, kv, d).transpose(2, 3) for x in (k, v))
        index_of = rows.int().view(1, B, 1, each).expand(L, B, kv, each).contiguous().to(DEV)
        shape = (L, B, kv, each, d)
    ko, vo = (torch.full(shape, 7.0, dtype=torch.bfloat16, device=DEV) for _ in range(2))
    with Ctx() as h:
        ta.ta_cache_append(h, c.struct(), batch, None, ta.view(kk, ragged), ta.view(vv, ragged), None, STREAM())
        ta.ta_cache_read(h, c.struct(), batch, index_of, ta.view(ko, ragged), ta.view(vo, ragged), STREAM())
        assert ta.ta_ctx_poll(h) == ta.TA_OK
    for x, got, old, name in ((k, ko, before[0], "k"), (v, vo, before[1], "v")):
        code, scale = codes(x.cpu().float(), form)
        want = code if scale is None else (code.float() * scale.unsqueeze(-1)).to(torch.bfloat16)
        got = got.cpu()
        got = got.transpose(1, 2) if ragged else got.transpose(2, 3).reshape(L, total, kv, d)
        assert torch.equal(got, want)
        now = held_rows(c, name, 42)
        now[:, seq.to(DEV), :, rows.to(DEV)] = old[:, seq.to(DEV), :, rows.to(DEV)]
        assert torch.equal(now, old)


@pytest.mark.parametrize("form", ["bf16", "e4m3", "int8"])
@pytest.mark.parametrize("d", [64, 128])
def test_gather_of_many_rows(form, d):
    L, B, kv, K, n = 2, 5, 4, 333, 1000
    g = torch.Generator().manual_seed(d)
    c = Cache(L, B, kv, d, 24, 42, form, "rows", seed=8)
    rows = torch.randint(0, n, (L, B, kv, K), generator=g, dtype=torch.int32)
    rows[torch.rand(rows.shape, generator=g) < 0.1] = -1
    ko, vo = (torch.full((L, B, kv, K, d), 7.0, dtype=torch.bfloat16, device=DEV) for _ in range(2))
    with Ctx() as h:
        ta.ta_cache_read(h, c.struct(), ta.make_batch(L, B, K, K, B * K), rows.to(DEV), ta.view(ko), ta.view(vo), STREAM())
        assert ta.ta_ctx_poll(h) == ta.TA_OK
    at = rows.clamp_min(0).long().to(DEV).unsqueeze(-1).expand(L, B, kv, K, d)
    for got, name in ((ko, "k"), (vo, "v")):
        want = torch.where(rows.to(DEV).unsqueeze(-1) < 0, 0.0, held_rows(c, name, n).gather(3, at))
        assert torch.equal(got, want.float().to(torch.bfloat16))


# ---- the rotation ----------------------------------------------------------------------------------------------------------------


@pytest.mark.parametrize("d,d_rot,layout,H,kv", [(128, 128, 0, 6, 2), (128, 64, 1, 4, 1), (64, 40, 0, 3, 1), (256, 256, 0, 1, 0), (8, 8, 1, 5, 0)])
@pytest.mark.parametrize("ragged", [True, False])
def test_several_tokens_a_thread(d, d_rot, layout, H, kv, ragged):
    B, L, each = 5, 2, 10001
    lens = [50, 0, 30000, 1, 19954] if ragged else [each] * B
    total = sum(lens)
    cu = torch.tensor([sum(lens[:i]) for i in range(B + 1)], dtype=torch.int32, device=DEV) if ragged else None
    batch = ta.make_batch(L, B, 0 if ragged else each, max(lens), total, cu)
    x = _randn(L, total, H + kv, d)
    q, k = x[:, :, :H], x[:, :, H:]
    qo, ko = torch.empty_like(q), torch.empty_like(k)
    if ragged:
        as_view = (lambda t: ta.view(t.transpose(1, 2), True))
    else:
        as_view = (lambda t: ta.ta_bf16_view(t.data_ptr(), t.stride(0), t.stride(1) * each, t.stride(2), t.stride(1)))
    rot, keep = rotary(d_rot, layout, magnitude=1.2)
    with Ctx() as h:
        ta.ta_rotate(h, batch, H, kv, d, rot, as_view(q), as_view(qo), as_view(k) if kv else ta.view(None),
                     as_view(ko) if kv else ta.view(None), STREAM())
        torch.cuda.synchronize()
        assert ta.ta_ctx_poll(h) == ta.TA_OK
    pos = torch.cat([torch.arange(n) for n in lens]).to(DEV).view(1, total, 1)
    for a, b in ((q, qo), (k, ko)):
        a = a.double()
        want = rotated(a, pos, frequencies(d_rot), d_rot, layout == 1, 1.2)
        if a.shape[2]:
            within(b.double(), want, U * want.abs() + 2.0 ** -20 * 1.2 * a.abs().amax(-1, keepdim=True) * 2, "rotate")
            assert torch.equal(b[..., d_rot:], a[..., d_rot:].to(torch.bfloat16))

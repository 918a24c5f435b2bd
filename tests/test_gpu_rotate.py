"""Rotary positions against a 64-bit statement: layouts, parts of a head, strides, positions, scalings, the inverse direction."""
import math

import pytest
import torch

import paper_2604_11288_b200 as ta
from decode_testlib import DEV, U, Ctx, frequencies, rotary, rotated, within

pytestmark = pytest.mark.gpu


def _tol(x, y, magnitude=1.0):
    # one rounding to bf16; the pair's products and sine and cosine in fp32: a few units of 2^-24 of |a| + |b|
    return U * y.abs() + 2.0 ** -20 * magnitude * x.abs().amax(-1, keepdim=True) * 2


def _run(q, k, batch, rot, d, ragged, inplace=False):
    qo = q if inplace else torch.full_like(q, 7.0)
    ko = k if inplace or k is None else torch.full_like(k, 7.0)
    v = (lambda t: ta.view(t, ragged))
    with Ctx() as h:
        ta.ta_rotate(h, batch, q.shape[-3], 0 if k is None else k.shape[-3], d, rot, v(q), v(qo), v(k), v(ko),
                     torch.cuda.current_stream().cuda_stream)
        torch.cuda.synchronize()
        assert ta.ta_ctx_poll(h) == ta.TA_OK
    return qo, ko


@pytest.mark.parametrize("d,d_rot", [(128, 128), (128, 64), (128, 104), (64, 64), (64, 40), (256, 256), (96, 72), (8, 8)])
@pytest.mark.parametrize("layout", [0, 1])
def test_uniform(d, d_rot, layout):
    g = torch.Generator().manual_seed(d + d_rot)
    L, B, n, H, kv = 2, 3, 5, 6, 2
    q, k = (torch.randn((L, B, n, h, d), generator=g).to(torch.bfloat16).to(DEV).transpose(2, 3) for h in (H, kv))
    pos = torch.randint(0, 131072, (B * n,), generator=g, dtype=torch.int32)
    rot, keep = rotary(d_rot, layout, positions=pos.to(DEV))
    qo, ko = _run(q, k, ta.make_batch(L, B, n, n, B * n), rot, d, False)
    f = frequencies(d_rot)
    for x, y in ((q, qo), (k, ko)):
        x = x.cpu().double()
        want = rotated(x, pos.view(B, 1, n), f, d_rot, layout == 1)
        within(y.cpu().double(), want, _tol(x, want), "rotate")
        assert torch.equal(y.cpu()[..., d_rot:], x[..., d_rot:].to(torch.bfloat16))


@pytest.mark.parametrize("lens", [[1], [0, 7, 0, 1, 300, 0], [2049, 1]])
@pytest.mark.parametrize("fused", [False, True])
def test_ragged_without_positions(lens, fused):
    g = torch.Generator().manual_seed(3)
    L, H, kv, d = 2, 5, 1, 128
    total = sum(lens)
    cu = torch.tensor([sum(lens[:i]) for i in range(len(lens) + 1)], dtype=torch.int32)
    if fused:  # queries, keys and values of a token side by side
        x = torch.randn((L, total, H + 2 * kv, d), generator=g).to(torch.bfloat16).to(DEV)
        q, k = x[:, :, :H].transpose(1, 2), x[:, :, H:H + kv].transpose(1, 2)
    else:
        q, k = (torch.randn((L, h, total, d), generator=g).to(torch.bfloat16).to(DEV) for h in (H, kv))
    before = (q.cpu().double(), k.cpu().double(), x.clone() if fused else None)
    rot, keep = rotary(d, 0)
    cu = cu.to(DEV)
    batch = ta.make_batch(L, len(lens), 0, max(lens), total, cu)
    qo, ko = _run(q, k, batch, rot, d, True, inplace=fused)
    pos = torch.cat([torch.arange(n) for n in lens])
    for x0, y in ((before[0], qo), (before[1], ko)):
        want = rotated(x0, pos, frequencies(d), d, False)
        within(y.cpu().double(), want, _tol(x0, want), "rotate")
    if fused:  # in place: the values beside them stay
        assert torch.equal(x[:, :, H + kv:], before[2][:, :, H + kv:])


def test_extreme_positions_lose_nothing():
    pos = torch.tensor([0, 1, -1, 2 ** 24 + 1, 2 ** 31 - 1, -2 ** 31, 999983, 131071], dtype=torch.int32)
    g = torch.Generator().manual_seed(4)
    q = torch.randn((1, 1, 3, len(pos), 128), generator=g).to(torch.bfloat16).to(DEV)
    rot, keep = rotary(128, 0, base=500000.0, positions=pos.to(DEV))
    qo, _ = _run(q, None, ta.make_batch(1, 1, len(pos), len(pos), len(pos)), rot, 128, False)
    # the angle from the same 64-bit turns, in whole numbers
    turns = [(int(p) * (int(t) % 2 ** 64)) % 2 ** 64 for p in pos for t in keep[0].cpu()]
    a = torch.tensor([t / 2.0 ** 64 for t in turns], dtype=torch.float64).view(len(pos), 64) * 2 * math.pi
    x = q.cpu().double()
    c, s = torch.cos(a), torch.sin(a)
    want = torch.cat((x[..., :64] * c - x[..., 64:] * s, x[..., :64] * s + x[..., 64:] * c), -1)
    within(qo.cpu().double(), want, _tol(x, want), "rotate")


@pytest.mark.parametrize("layout", [0, 1])
def test_inverse_undoes_and_is_the_gradient(layout):
    g = torch.Generator().manual_seed(5)
    n, d, d_rot, mag = 33, 128, 96, 1.25
    x, grad = (torch.randn((1, 1, 4, n, d), generator=g).to(torch.bfloat16).to(DEV) for _ in range(2))
    batch = ta.make_batch(1, 1, n, n, n)
    fwd, k1 = rotary(d_rot, layout, magnitude=mag)
    bwd, k2 = rotary(d_rot, layout, magnitude=mag, inverse=True)
    undo, k3 = rotary(d_rot, layout, magnitude=1 / mag, inverse=True)
    y, _ = _run(x, None, batch, fwd, d, False)
    dx, _ = _run(grad, None, batch, bwd, d, False)
    want = rotated(grad.cpu().double(), torch.arange(n), frequencies(d_rot), d_rot, layout == 1, mag, True)
    within(dx.cpu().double(), want, _tol(grad.cpu().double(), want, mag), "gradient")
    back, _ = _run(y, None, batch, undo, d, False)
    top = x.cpu().double().abs().amax(-1, keepdim=True)
    within(back.cpu().double(), x.cpu().double(), 3 * U * 2 * top, "undone")  # rounded twice
    # differences: the map is linear, so a step of 64 in one coordinate gives 64 times a column of the matrix
    for c in (0, 5, d_rot // 2, d_rot - 1, d - 1):
        lo, hi = x.clone(), x.clone()
        lo[..., c], hi[..., c] = -32.0, 32.0
        step = (_run(hi, None, batch, fwd, d, False)[0].cpu().double() - _run(lo, None, batch, fwd, d, False)[0].cpu().double()) / 64
        unit = torch.zeros((1, 1, d, n, d), dtype=torch.bfloat16, device=DEV)  # head j: output coordinate j
        unit[0, 0, torch.arange(d), :, torch.arange(d)] = 1.0
        rows = _run(unit, None, batch, bwd, d, False)[0].cpu().double()[0, 0, :, :, c]  # d out_j / d x_c for every position
        # two roundings of values up to 1.25 (32 + 5) and the row's own
        within(step[0, 0], rows.T.unsqueeze(0).expand(4, n, d), torch.full((4, n, d), 2 * U * 48 / 64 + 2 * U, dtype=torch.float64), "difference")


def test_scaling_tables():
    d_rot, base, factor, orig = 128, 500000.0, 8.0, 8192.0
    f = frequencies(d_rot, base)
    got = {}
    for kind in range(5):
        phase = torch.empty(d_rot // 2, dtype=torch.int64)
        got[kind] = (ta.ta_rotary_table(d_rot, base, kind, factor, orig, 1.0, 4.0, phase), phase.double() / 2.0 ** 64 * 2 * math.pi)
    rel, low = 1e-12, 2 * math.pi * 2.0 ** -64  # two roundings of pow in 64 bits; turns are whole multiples of 2^-64
    assert torch.allclose(got[0][1], f, rtol=rel, atol=low) and torch.allclose(got[1][1], f / factor, rtol=rel, atol=low)
    assert torch.allclose(got[2][1], frequencies(d_rot, base * factor ** (128 / 126)), rtol=rel, atol=low)
    turns = orig * f / (2 * math.pi)
    w = ((turns - 1.0) / 3.0).clamp(0, 1)
    assert torch.allclose(got[4][1], w * f + (1 - w) * f / factor, rtol=rel, atol=low)
    assert (got[3][1] <= f * (1 + rel)).all() and (got[3][1] >= f / factor * (1 - rel) - low).all()
    assert (got[3][1][turns > 4.5] == got[0][1][turns > 4.5]).all() and (got[3][1][turns < 0.5] < f[turns < 0.5] / factor * 1.001).all()
    assert abs(got[3][0] - (0.1 * math.log(factor) + 1)) < 1e-6 and all(got[k][0] == 1.0 for k in (0, 1, 2, 4))


def test_refusals():
    q = torch.zeros((1, 1, 2, 4, 128), dtype=torch.bfloat16, device=DEV)
    v, none = ta.view(q), ta.view(None)
    batch = ta.make_batch(1, 1, 4, 4, 4)
    good, keep = rotary(128)

    def status(rot=good, d=128, Hq=2, Hkv=0, a=v, b=v, k=none, bt=batch):
        with pytest.raises(ta.TAError) as e:
            ta.ta_rotate(h, bt, Hq, Hkv, d, rot, a, b, k, k)
        return e.value.status

    with Ctx() as h:
        assert status(None) == ta.TA_ERR_INVALID_ARG
        assert status(rotary(128, layout=2)[0]) == ta.TA_ERR_INVALID_ARG
        assert status(rotary(128, magnitude=math.inf)[0]) == ta.TA_ERR_INVALID_ARG
        assert status(ta.make_rotary(None, 128)) == ta.TA_ERR_INVALID_ARG
        assert status(ta.make_rotary(keep[0], 12)) == ta.TA_ERR_UNSUPPORTED  # no multiple of 8
        assert status(ta.make_rotary(keep[0], 136)) == ta.TA_ERR_INVALID_ARG  # more than the head
        assert status(d=264) == ta.TA_ERR_UNSUPPORTED and status(d=100) == ta.TA_ERR_UNSUPPORTED
        assert status(Hq=0) == ta.TA_ERR_INVALID_ARG and status(Hkv=2) == ta.TA_ERR_INVALID_ARG  # no keys
        assert status(a=ta.ta_bf16_view(q.data_ptr() + 2, 1024, 1024, 512, 128)) == ta.TA_ERR_ALIGNMENT
        assert status(a=ta.ta_bf16_view(q.data_ptr(), 1024, 1024, 512, 120)) == ta.TA_ERR_INVALID_ARG
        assert status(bt=ta.make_batch(1, 1, 4, 4, 5)) == ta.TA_ERR_INVALID_ARG
        assert ta.ta_ctx_poll(h) == ta.TA_OK
    with pytest.raises(ta.TAError):
        ta.ta_rotate(None, batch, 2, 0, 128, good, v, v, none, none)
    phase = torch.empty(64, dtype=torch.int64)
    for bad in ((127, 1e4, 0, 1, 0, 0, 0), (128, 1.0, 0, 1, 0, 0, 0), (128, 1e4, 5, 1, 0, 0, 0), (128, 1e4, 1, 0.5, 0, 0, 0),
                (128, 1e4, 3, 2.0, 4096, 32.0, 1.0), (128, 1e4, 4, 2.0, 0.0, 1.0, 4.0), (2, 1e4, 2, 2.0, 0, 0, 0),
                (128, math.nan, 0, 1, 0, 0, 0)):
        with pytest.raises(ta.TAError):
            ta.ta_rotary_table(*bad, phase)


def test_nothing_to_do():
    q = torch.zeros((1, 1, 2, 1, 128), dtype=torch.bfloat16, device=DEV)
    rot, keep = rotary(128)
    with Ctx() as h:
        ta.ta_rotate(h, ta.make_batch(1, 1, 0, 0, 0), 2, 0, 128, rot, ta.view(q), ta.view(q), ta.view(None), ta.view(None))
        assert ta.ta_ctx_poll(h) == ta.TA_OK

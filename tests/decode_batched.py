"""The 64-bit statements of decode_testlib for calls of thousands of units: all of them at once, on the device."""
import math

import torch

from decode_testlib import DEV, U


def held_rows(c, name, n):
    """Rows 0..n-1 of every unit of a Cache in 64 bits: [L, B, kv, n, d]."""
    ids = torch.stack([c.page_ids(b) for b in range(c.B)]).to(DEV)
    x, s = c.dev[name], c.dev[name + "_scale"]
    raw = (x.view(torch.int8) if x.element_size() == 1 else x)[:, ids].contiguous().view(x.dtype)  # [L, B, wide, kv, page, d]
    y = raw.float().double()
    if s is not None:
        y = y * s[:, ids].double().unsqueeze(-1)
    return y.transpose(2, 3).reshape(c.L, c.B, c.kv, c.wide * c.page, c.d)[..., :n, :]


def rotated(x, positions, f, d_rot, interleaved, magnitude=1.0, inverse=False):
    """decode_testlib.rotated with broadcast positions, on x's device."""
    a = positions.to(x.device).double().unsqueeze(-1) * f.to(x.device)
    c, s = magnitude * torch.cos(a), magnitude * torch.sin(a) * (-1 if inverse else 1)
    i = torch.arange(d_rot // 2, device=x.device)
    m, n = (2 * i, 2 * i + 1) if interleaved else (i, i + d_rot // 2)
    y = x.clone()
    y[..., m], y[..., n] = x[..., m] * c - x[..., n] * s, x[..., m] * s + x[..., n] * c
    return y


def attend(c, q, T, lens, causal=True, rot=None):
    """q [L, B, Hq, T, d] in bf16 on the device, lens [L, B, kv]. out, lse, mass and their tolerances, as attend_reference has them;
    rot = (f, d_rot, interleaved, magnitude, positions [B, T] or None)."""
    L, B, H, _, d = q.shape
    G, n = H // c.kv, max(1, int(lens.max()))
    lens = lens.to(DEV)
    x = q.double().view(L, B, c.kv, G, T, d)
    t = torch.arange(T, device=DEV)
    if rot is not None:
        f, d_rot, inter, magnitude, pos = rot
        at = lens[..., None, None] - T + t if pos is None else pos.to(DEV).view(1, B, 1, 1, T)
        x = rotated(x, at.expand(L, B, c.kv, 1, T), f, d_rot, inter, magnitude)
    k, v = held_rows(c, "k", n), held_rows(c, "v", n)
    seen = lens[..., None] - (T - 1 - t if causal else 0 * t)                         # [L, B, kv, T]
    there = torch.arange(n, device=DEV) < seen[..., None]                             # [L, B, kv, T, n]
    there = there.unsqueeze(3)
    s = torch.einsum("lbgqtd,lbgnd->lbgqtn", x, k) / math.sqrt(d)
    A = torch.einsum("lbgqtd,lbgnd->lbgqtn", x.abs(), k.abs()) / math.sqrt(d)
    A = torch.where(there, A, 0.0).amax(-1)
    lse = torch.logsumexp(torch.where(there, s, -math.inf), -1)
    p = torch.where(there & (lse > -math.inf).unsqueeze(-1), torch.exp(s - lse.nan_to_num(0.0, 0.0, 0.0).unsqueeze(-1)), 0.0)
    rel = 2.0 ** -18 * A + 2.0 ** -14
    out = torch.einsum("lbgqtn,lbgnd->lbgqtd", p, v)
    tol = U * out.abs() + rel.unsqueeze(-1) * torch.einsum("lbgqtn,lbgnd->lbgqtd", p, v.abs()) + 1e-30
    mass, mass_tol = p.sum((3, 4)), (p * rel.unsqueeze(-1)).sum((3, 4)) + 2.0 ** -126
    return [y.cpu() for y in (out.view(L, B, H, T, d), lse.view(L, B, H, T), mass, tol.view(L, B, H, T, d), rel.view(L, B, H, T), mass_tol)]

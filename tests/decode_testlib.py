"""Plain 64-bit statements of the decode loop's operators, and the tolerances of their tests.

Tolerances follow from the formats, before any run. bf16 has 8 significant bits: rounding costs at most U = 2^-8 of the value.
Kernels sum in fp32 (2^-24 a rounding, twice that where a tensor core truncates): a score of d <= 128 products is off by at
most 2^-19 A with A = scale * sum |q k|, counting the rotation's and the scale's roundings in; a probability keeps 16 bits
and is off by at most (2^-18 A + 2^-14) of itself (its own score, the normaliser's, exponential, rounding to two bf16 parts,
sums over rows), an output by that share of sum p |v|, besides its own rounding."""
from __future__ import annotations

import math

import torch

import paper_2604_11288_b200 as ta

U = 2.0 ** -8
DEV = "cuda:0"
FULL = {"e4m3": 448.0, "int8": 127.0}
TYPES = {"bf16": torch.bfloat16, "e4m3": torch.float8_e4m3fn, "int8": torch.int8}


def frequencies(d_rot, base=10000.0):
    return torch.tensor([base ** (-2.0 * i / d_rot) for i in range(d_rot // 2)], dtype=torch.float64)


def rotated(x, positions, f, d_rot, interleaved, magnitude=1.0, inverse=False):
    """x [..., n, d] in 64 bits, positions broadcastable to [..., n]."""
    a = positions.double().unsqueeze(-1) * f
    c, s = magnitude * torch.cos(a), magnitude * torch.sin(a) * (-1 if inverse else 1)
    y = x.clone()
    i = torch.arange(d_rot // 2)
    m, n = (2 * i, 2 * i + 1) if interleaved else (i, i + d_rot // 2)
    y[..., m], y[..., n] = x[..., m] * c - x[..., n] * s, x[..., m] * s + x[..., n] * c
    return y


def rotary(d_rot, layout=0, base=10000.0, scaling=None, magnitude=None, inverse=False, positions=None):
    """A ta_rotary with its tensors (keep the second value)."""
    phase = torch.empty(d_rot // 2, dtype=torch.int64)
    m = ta.ta_rotary_table(d_rot, base, *(scaling or (ta.TA_SCALING_PLAIN, 1.0, 0.0, 0.0, 0.0)), phase)
    phase = phase.to(DEV)
    return ta.make_rotary(phase, d_rot, layout, m if magnitude is None else magnitude, inverse, positions), (phase, positions)


def codes(x, form):
    """The documented codes and scales of fp32 rows, in 32 bits."""
    if form == "bf16":
        return x.to(torch.bfloat16), None
    bad = ~torch.isfinite(x).all(-1, keepdim=True)
    m = torch.where(bad, torch.ones_like(x[..., :1]), x.abs().amax(-1, keepdim=True).clamp_min(2.0 ** -100))
    y = torch.where(bad, torch.zeros_like(x), x * torch.div(torch.full_like(m, FULL[form]), m))
    c = y.round() if form == "int8" else y.clamp(-448.0, 448.0)
    return c.to(TYPES[form]), torch.where(bad, torch.full_like(m, math.nan), m / FULL[form])[..., 0]


class Cache:
    """A cache on the device, its rows and table as CPU tensors in 64 bits too."""

    def __init__(self, L=1, B=1, kv=1, d=128, page=16, pages_per_seq=4, form="bf16", order="heads", dense=False, seed=0, lens=None,
                 len_uniform=0, scale=1.0, spare=3):
        g = torch.Generator().manual_seed(seed)
        self.L, self.B, self.kv, self.d, self.page, self.wide, self.form = L, B, kv, d, page, pages_per_seq, form
        self.pages = B * pages_per_seq + (0 if dense else spare)
        shape = (L, self.pages, kv, page, d)
        self.stored, self.scales = {}, {}
        perm = (0, 1, 3, 2, 4) if order == "rows" else (0, 1, 2, 3, 4)
        self.dev = {}
        for name in ("k", "v"):
            x = torch.randn(shape, generator=g) * scale
            c, s = codes(x.to(torch.bfloat16).float(), form)
            self.put(name, c, s, perm)
        self.table = None if dense else torch.randperm(self.pages, generator=g)[:B * pages_per_seq].view(B, pages_per_seq).int()
        self.d_table = None if dense else self.table.to(DEV)
        self.lens = lens
        self.d_lens = None if lens is None else torch.tensor(lens, dtype=torch.int32).to(DEV)
        self.len_uniform = len_uniform
        self.order = perm

    def put(self, name, c, s, perm):
        raw = c.view(torch.int8) if c.element_size() == 1 else c
        self.dev[name] = raw.permute(perm).contiguous().to(DEV).permute(perm).view(c.dtype)
        self.dev[name + "_scale"] = None if s is None else s.permute(perm[:4]).contiguous().to(DEV).permute(perm[:4])

    def struct(self):
        return ta.make_cache(self.dev["k"], self.dev["v"], self.dev["k_scale"], self.dev["v_scale"], table=self.d_table, batch=self.B,
                             lens=self.d_lens, len_uniform=self.len_uniform)

    def page_ids(self, b):
        return torch.arange(self.wide) + b * self.wide if self.table is None else self.table[b].long()

    def rows(self, name, l, b, g, n):
        """Rows 0..n-1 of a unit in 64 bits, as the device holds them."""
        c = self.dev[name]
        raw = (c.view(torch.int8) if c.element_size() == 1 else c).cpu()
        ids = self.page_ids(b)[:max(1, -(-n // self.page))]
        x = raw[l, ids, g].contiguous().view(c.dtype).float().double().reshape(-1, self.d)[:n]
        if self.dev[name + "_scale"] is not None:
            x = x * self.dev[name + "_scale"].cpu()[l, ids, g].double().reshape(-1, 1)[:n]
        return x

    def len_of(self, l, b, g):
        if self.lens is None:
            return self.len_uniform
        v = self.lens[l] if isinstance(self.lens[0], list) else None
        return v[b][g] if v is not None else self.lens[b]


class Ctx:
    def __init__(self, scratch=1 << 20):
        self.h = ta.ta_ctx_create(0, scratch)

    def __enter__(self):
        return self.h

    def __exit__(self, *_):
        ta.ta_ctx_destroy(self.h)


def attend_reference(c: Cache, q, T, new_rows=0, causal=True, scale=0.0, rot=None):
    """q [L, B, Hq, T, d] CPU. Returns out, lse, mass, and tolerances of out, lse and mass; rot = (f, d_rot, interleaved, magnitude,
    inverse, positions [B, T] or None)."""
    L, B, H, _, d = q.shape
    G = H // c.kv
    scale = scale or 1.0 / math.sqrt(d)
    n_max = max(1, max(c.len_of(l, b, g) + new_rows for l in range(L) for b in range(B) for g in range(c.kv)))
    out, tol = torch.zeros(L, B, H, T, d, dtype=torch.float64), torch.zeros(L, B, H, T, d, dtype=torch.float64)
    lse, lse_tol = torch.full((L, B, H, T), -math.inf, dtype=torch.float64), torch.zeros(L, B, H, T, dtype=torch.float64)
    mass, mass_tol = torch.zeros(L, B, c.kv, n_max, dtype=torch.float64), torch.zeros(L, B, c.kv, n_max, dtype=torch.float64)
    for l in range(L):
        for b in range(B):
            for g in range(c.kv):
                n = max(0, c.len_of(l, b, g) + new_rows)
                k, v = c.rows("k", l, b, g, n), c.rows("v", l, b, g, n)
                for t in range(T):
                    seen = n - (T - 1 - t) if causal else n
                    if seen <= 0:
                        continue
                    x = q[l, b, g * G:(g + 1) * G, t].double()
                    if rot is not None:
                        f, d_rot, inter, mag, inv, pos = rot
                        p = torch.tensor([n - T + t if pos is None else int(pos[b][t])])
                        x = rotated(x.unsqueeze(1), p, f, d_rot, inter, mag, inv)[:, 0]
                    s = scale * x @ k[:seen].T
                    A = (scale * x.abs() @ k[:seen].abs().T).amax(-1, keepdim=True)
                    lse[l, b, g * G:(g + 1) * G, t] = torch.logsumexp(s, -1)
                    p = torch.softmax(s, -1)
                    rel = 2.0 ** -18 * A + 2.0 ** -14
                    out[l, b, g * G:(g + 1) * G, t] = p @ v[:seen]
                    tol[l, b, g * G:(g + 1) * G, t] = U * (p @ v[:seen]).abs() + rel * (p @ v[:seen].abs()) + 1e-30
                    lse_tol[l, b, g * G:(g + 1) * G, t] = rel[:, 0]
                    mass[l, b, g, :seen] += p.sum(0)
                    mass_tol[l, b, g, :seen] += (p * rel).sum(0) + 2.0 ** -126  # below fp32's normal numbers nothing is kept
    return out, lse, mass, tol, lse_tol, mass_tol


def run_attend(c: Cache, q_dev, T, new_rows=0, max_len=None, causal=True, scale=0.0, rot=None, with_mass=True, mass_stride=None,
               out=None, stream=None, ctx=None):
    """Through the library: out, lse, mass (CPU, 64 bits), with guard values behind the outputs checked."""
    L, B, H, _, d = q_dev.shape
    s = c.struct()
    max_len = c.wide * c.page if max_len is None else max_len
    mass_stride = max_len if mass_stride is None else mass_stride
    out = torch.full((L + 1, B, H, T, d), 7.0, dtype=torch.bfloat16, device=DEV) if out is None else out
    lse = torch.full((L + 1, B, H, T), 7.0, device=DEV)
    mass = torch.full((L + 1, B, c.kv, mass_stride), 7.0, device=DEV) if with_mass else None
    need = ta.ta_attend_scratch_bytes(s, H, T, max_len, with_mass)
    own = ctx is None
    h = ta.ta_ctx_create(0, need) if own else ctx
    try:
        ta.ta_attend(h, s, H, T, new_rows, max_len, causal, scale, rot, ta.view(q_dev), ta.view(out[:L]), lse, mass,
                     mass_stride if with_mass else 0, stream if stream is not None else torch.cuda.current_stream().cuda_stream)
        torch.cuda.synchronize()
        if own:
            assert ta.ta_ctx_poll(h) == ta.TA_OK
    finally:
        if own:
            ta.ta_ctx_destroy(h)
    assert (out[L:] == 7.0).all() and (lse[L:] == 7.0).all()
    if with_mass:
        assert (mass[L:] == 7.0).all()
    return out[:L].cpu().double(), lse[:L].cpu().double(), None if mass is None else mass[:L].cpu().double()


def within(got, want, tol, what):
    bad = ~((got == want) | ((got - want).abs() <= tol))
    assert not bad.any(), (what, int(bad.sum()), got[bad][:4], want[bad][:4], tol[bad][:4])

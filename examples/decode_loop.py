"""A decode loop over a retained cache: compress a prompt, then generate with one eviction decision per token.

    python examples/decode_loop.py [--format bf16|e4m3|int8] [--steps N] [--budget K] [--tokens N]

There is no model here: queries, keys and values are drawn from a seed where a model's projections would stand. Everything
between them is the library's:

  prompt   ta_rotate        queries and keys to their positions
           ta_compress      which K tokens of every head stay, gathered
           ta_cache_append  the retained rows into a cache of K + 1 rows per head, in the cache's format
  token    ta_cache_append  the new key, rotated on its way, and value into the row that the last eviction freed
           ta_attend        the new query, rotated on its way, over the rows: output and attention mass per row
           ta_stream_step   the mass decides which token goes
"""
from __future__ import annotations

import argparse
import os
import sys
import time

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2604_11288_b200 as ta  # noqa: E402

DTYPES = {"bf16": torch.bfloat16, "e4m3": torch.float8_e4m3fn, "int8": torch.int8}
BASE = 500000.0


class DecodeLoop:
    def __init__(self, n=4096, layers=4, batch=2, Hq=32, Hkv=8, d=128, K=64, form="bf16", vocab=32000, seed=0, device="cuda:0"):
        self.n, self.L, self.B, self.Hq, self.Hkv, self.d, self.K, self.dev = n, layers, batch, Hq, Hkv, d, K, torch.device(device)
        self.gen = torch.Generator(device=device)
        self.gen.manual_seed(seed)
        self.vocab = vocab
        self.pol = ta.ta_policy_default(ta.TA_PRESET_THEOREM, K)
        self.pol.vocab_size = vocab
        self.key_ids = [11, 12]  # the anchor pattern, "key :" say
        # ---- the prompt: ids with one anchor and its value in every sequence, queries of the last rows, keys, values
        self.ids = torch.randint(100, vocab, (batch, n), generator=self.gen, device=device, dtype=torch.int32)
        self.anchor = n // 3
        self.ids[:, self.anchor:self.anchor + 2] = torch.tensor(self.key_ids, dtype=torch.int32, device=device)
        W = self.pol.obs_window  # (of a shorter prompt the first rows are not looked at)
        q, k, self.v = self._randn(layers, batch, Hq, W, d), self._randn(layers, batch, Hkv, n, d), self._randn(layers, batch, Hkv, n, d)
        # ---- handles that the whole loop keeps
        self.prompt = ta.make_batch(layers, batch, n, n, batch * n)
        self.one = ta.make_batch(layers, batch, 1, 1, batch)
        dtype, rows = DTYPES[form], K + 1
        self.k_rows, self.v_rows = (torch.zeros((layers, batch, Hkv, rows, d), dtype=dtype, device=device) for _ in range(2))
        self.k_scale, self.v_scale = ((None, None) if form == "bf16" else
                                      (torch.zeros((layers, batch, Hkv, rows), device=device) for _ in range(2)))
        self.cache = ta.make_cache(self.k_rows, self.v_rows, self.k_scale, self.v_scale, batch=batch)  # a page per sequence
        self._stream_state()
        scratch = max(ta.ta_scratch_bytes(self.prompt, Hq, Hkv, d, K, self.pol), ta.ta_stream_scratch_bytes(self.st),
                      ta.ta_attend_scratch_bytes(self.cache, Hq, 1, rows, True))
        self.ctx = ta.ta_ctx_create(self.dev.index or 0, scratch)
        self.pats = ta.ta_patterns_create(self.ctx, [self.key_ids])
        phase = torch.empty(d // 2, dtype=torch.int64)
        magnitude = ta.ta_rotary_table(d, BASE, ta.TA_SCALING_PLAIN, 1.0, 0.0, 0.0, 0.0, phase)
        self.phase = phase.to(device)
        self.positions = torch.empty(batch, dtype=torch.int32, device=device)  # of the new token
        self.rot_prompt = ta.make_rotary(self.phase, d, magnitude=magnitude)
        self.rot_window = ta.make_rotary(self.phase, d, magnitude=magnitude,
                                         positions=self._keep(torch.arange(n - W, n, dtype=torch.int32, device=device).repeat(batch)))
        self.rot_token = ta.make_rotary(self.phase, d, magnitude=magnitude, positions=self.positions)
        self.mass = torch.zeros((layers, batch, Hkv, rows), device=device)
        self.out = torch.zeros((layers, batch, Hq, 1, d), dtype=torch.bfloat16, device=device)
        self.lse = torch.zeros((layers, batch, Hq, 1), device=device)
        self.evicted = torch.zeros(layers * batch * Hkv, dtype=torch.int32, device=device)
        self._prefill(q, k, W)

    def _keep(self, t):
        self._held = getattr(self, "_held", []) + [t]
        return t

    def _randn(self, *shape):
        return torch.randn(shape, generator=self.gen, dtype=torch.bfloat16, device=self.dev)

    def _stream_state(self):
        U, rows, B = self.L * self.B * self.Hkv, self.K + 1, self.B
        z = (lambda *s, dt=torch.int32: torch.zeros(s, dtype=dt, device=self.dev))
        self.s = dict(pos=z(U, rows), slot=z(U, rows), tok=z(U, rows), A=z(U, rows, dt=torch.float32), P=z(U, rows, dt=torch.float32),
                      V=z(U, rows, dt=torch.float32), S=z(U, rows, dt=torch.uint8), next_slot=z(U), n_seen=z(B),
                      hist=z(B, self.vocab), tok_ring=z(B, 8), anc_B=z(B, 64, dt=torch.float32), anc_L=z(B, 64))
        self.st = ta.ta_stream(self.L, self.B, self.Hkv, self.K, 0, *[t.data_ptr() for t in self.s.values()])

    def _prefill(self, q, k, W):
        L, B, Hkv, K, d, n = self.L, self.B, self.Hkv, self.K, self.d, self.n
        stream = torch.cuda.current_stream().cuda_stream
        none, window = ta.view(None), ta.make_batch(L, B, W, W, B * W)
        ta.ta_rotate(self.ctx, self.prompt, Hkv, 0, d, self.rot_prompt, ta.view(k), ta.view(k), none, none, stream)
        ta.ta_rotate(self.ctx, window, self.Hq, 0, d, self.rot_window, ta.view(q), ta.view(q), none, none, stream)
        k_out, v_out = (torch.empty((L, B, Hkv, K, d), dtype=torch.bfloat16, device=self.dev) for _ in range(2))
        idx = torch.empty((L, B, Hkv, K), dtype=torch.int32, device=self.dev)
        count = torch.empty((L, B, Hkv), dtype=torch.int32, device=self.dev)
        ta.ta_compress(self.ctx, self.pats, self.pol, self.prompt, self.Hq, Hkv, d, K, self.ids, ta.view(q), ta.view(k), ta.view(self.v),
                       0, k_out, v_out, idx, count, stream)
        kept = min(K, n)
        rows = torch.where(idx >= 0, torch.arange(K, device=self.dev, dtype=torch.int32), -1).to(torch.int32).contiguous()
        ta.ta_cache_append(self.ctx, self.cache, ta.make_batch(L, B, K, K, B * K), None, ta.view(k_out), ta.view(v_out), rows, stream)
        # the decode loop's state: retained rows in position order, everything that was seen counted
        flags = torch.empty(B * n, dtype=torch.uint8, device=self.dev)
        V, u = torch.empty(B * n, device=self.dev), torch.empty(B * n, device=self.dev)
        ta.ta_sponsor_mask(self.ctx, self.pats, self.pol, self.prompt, self.ids, flags, V, u, stream)
        U, at = L * B * Hkv, idx.view(L, B, Hkv * K).long().clamp_min(0)
        pick = (lambda t: torch.gather(t.view(1, B, n).expand(L, B, n), 2, at).view(U, K))
        s = self.s
        s["pos"][:, :K], s["slot"][:, :K] = idx.view(U, K).clamp_min(0), torch.arange(K, device=self.dev, dtype=torch.int32)
        s["tok"][:, :K], s["V"][:, :K] = pick(self.ids.view(-1)), pick(V)
        s["S"][:, :K] = (pick(flags) & ta.TA_FLAG_ANCHOR_TOKEN).to(torch.uint8)
        s["next_slot"].fill_(kept)
        s["n_seen"].fill_(n)
        for b in range(B):
            s["hist"][b] = torch.bincount(self.ids[b].long(), minlength=self.vocab).to(torch.int32)
        last = torch.arange(max(0, n - 8), n, device=self.dev)
        s["tok_ring"][:, last % 8] = self.ids[:, last]
        self.st.cache_len = kept
        self.retained = idx
        torch.cuda.current_stream().synchronize()  # what this function made is gone after it
        assert ta.ta_ctx_poll(self.ctx) == ta.TA_OK

    def step(self, new_ids, q, k, v):
        """One token per sequence. q [L, B, Hq, 1, d], k and v [L, B, Hkv, 1, d], not rotated; the output is self.out."""
        stream = torch.cuda.current_stream().cuda_stream
        held = self.st.cache_len
        self.positions.copy_(self.s["n_seen"])
        ta.ta_cache_append(self.ctx, self.cache, self.one, self.rot_token, ta.view(k), ta.view(v), self.s["next_slot"], stream)
        self.cache.len_uniform = held
        ta.ta_attend(self.ctx, self.cache, self.Hq, 1, 1, self.K + 1, True, 0.0, self.rot_token, ta.view(q), ta.view(self.out), self.lse,
                     self.mass, self.K + 1, stream)
        ta.ta_stream_step(self.ctx, self.pats, self.pol, self.st, new_ids, self.mass, self.evicted, stream)

    def random_step(self):
        ids = torch.randint(100, self.vocab, (self.B,), generator=self.gen, device=self.dev, dtype=torch.int32)
        q, k, v = self._randn(self.L, self.B, self.Hq, 1, self.d), self._randn(self.L, self.B, self.Hkv, 1, self.d), \
            self._randn(self.L, self.B, self.Hkv, 1, self.d)
        self.step(ids, q, k, v)
        return ids, q, k, v

    def sponsored_left(self):
        """How many heads still hold the first token behind the prompt's anchor."""
        value = self.anchor + 2
        return int((self.s["pos"][:, :self.st.cache_len] == value).any(1).sum()), self.L * self.B * self.Hkv

    def close(self):
        ta.ta_patterns_destroy(self.pats)
        ta.ta_ctx_destroy(self.ctx)


def main():
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--format", choices=sorted(DTYPES), default="bf16")
    ap.add_argument("--steps", type=int, default=200)
    ap.add_argument("--budget", type=int, default=256)
    ap.add_argument("--tokens", type=int, default=4096)
    ap.add_argument("--layers", type=int, default=32)
    ap.add_argument("--batch", type=int, default=4)
    a = ap.parse_args()
    loop = DecodeLoop(n=a.tokens, layers=a.layers, batch=a.batch, K=a.budget, form=a.format)
    try:
        for _ in range(5):
            loop.random_step()
        torch.cuda.synchronize()
        t = time.perf_counter()
        for _ in range(a.steps):
            loop.random_step()
        torch.cuda.synchronize()
        took = time.perf_counter() - t
        assert ta.ta_ctx_poll(loop.ctx) == ta.TA_OK
        held, of = loop.sponsored_left()
        print(f"{a.steps} tokens x {a.batch} sequences x {a.layers} layers, {a.budget} of {a.tokens} rows per head in {a.format}: "
              f"{took / a.steps * 1e6:.0f} us a token; the anchor's value is still held by {held} of {of} heads")
    finally:
        loop.close()


if __name__ == "__main__":
    main()

"""The decode loop of examples/decode_loop.py: every step's output, mass and eviction against plain statements."""
import math
import os
import sys

import numpy as np
import pytest
import torch

import oracle
import paper_2604_11288_b200 as ta
from decode_testlib import U, frequencies, rotated, within
from oracle.ta_stream_oracle import StreamOracle
from ta_testlib import oracle_policy

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))
from decode_loop import BASE, DecodeLoop  # noqa: E402

pytestmark = pytest.mark.gpu


def _held(loop, name, unit):
    """Rows of a unit in 64 bits, as the cache holds them."""
    rows = {"k": loop.k_rows, "v": loop.v_rows}[name].view(-1, loop.K + 1, loop.d)[unit].float().double()
    scale = {"k": loop.k_scale, "v": loop.v_scale}[name]
    return (rows if scale is None else rows * scale.view(-1, loop.K + 1)[unit].double().unsqueeze(-1)).cpu()


@pytest.mark.parametrize("form", ["bf16", "e4m3", "int8"])
@pytest.mark.parametrize("n,K", [(300, 24), (24, 24), (17, 24)])
def test_steps(form, n, K):
    loop = DecodeLoop(n=n, layers=2, batch=2, Hq=8, Hkv=2, K=K, form=form, vocab=500, seed=n)
    f = frequencies(loop.d, BASE)
    try:
        for _ in range(K + 6):
            before = {x: loop.s[x].cpu().clone() for x in ("pos", "slot", "next_slot", "n_seen")}
            held = loop.st.cache_len
            ids, q, k, v = loop.random_step()
            torch.cuda.synchronize()
            assert ta.ta_ctx_poll(loop.ctx) == ta.TA_OK
            after = {x: loop.s[x].cpu() for x in ("pos", "slot", "next_slot", "n_seen")}
            for unit in range(loop.L * loop.B * loop.Hkv):
                g, b, l = unit % loop.Hkv, unit // loop.Hkv % loop.B, unit // loop.Hkv // loop.B
                new, pos = int(before["next_slot"][unit]), int(before["n_seen"][b])
                # the new row is the rotated key, in the cache's format
                x = k[l, b, g, 0].cpu().double()
                want = rotated(x.unsqueeze(0), torch.tensor([pos]), f, loop.d, False)[0]
                top = want.abs().max()
                step = {"bf16": U * want.abs(), "int8": top / 254 * torch.ones_like(want),
                        "e4m3": torch.maximum(want.abs() * 2.0 ** -4, top / 448 * 2.0 ** -10)}[form]
                keys, vals = _held(loop, "k", unit), _held(loop, "v", unit)
                within(keys[new], want, step * 1.01 + 2.0 ** -19 * x.abs().max(), "row")
                # the attention over the rows that are there
                rows = torch.cat((before["slot"][unit, :held], torch.tensor([new], dtype=torch.int32))).long()
                assert len(set(rows.tolist())) == held + 1 and int(rows.max()) <= held
                y = rotated(q[l, b, 4 * g:4 * g + 4, 0].cpu().double().unsqueeze(1), torch.tensor([pos]), f, loop.d, False)[:, 0]
                s = y @ keys[:held + 1].T / math.sqrt(loop.d)
                A = (y.abs() @ keys[:held + 1].abs().T / math.sqrt(loop.d)).amax(-1, keepdim=True)
                p = torch.softmax(s, -1)
                rel = 2.0 ** -18 * A + 2.0 ** -14
                o = p @ vals[:held + 1]
                within(loop.out[l, b, 4 * g:4 * g + 4, 0].cpu().double(), o, U * o.abs() + rel * (p @ vals[:held + 1].abs()), "out")
                within(loop.mass.view(-1, K + 1)[unit].cpu().double()[:held + 1], p.sum(0), (p * rel).sum(0), "mass")
                assert (loop.mass.view(-1, K + 1)[unit][held + 1:] == 0).all()
                # what goes frees its row for the next token
                if held == K:
                    out_pos = int(loop.evicted[unit])
                    gone = (before["pos"][unit, :held] == out_pos).nonzero()
                    row = int(before["slot"][unit, gone[0, 0]]) if len(gone) else new
                    assert int(after["next_slot"][unit]) == row and out_pos not in after["pos"][unit, :K].tolist()
                else:
                    assert int(loop.evicted[unit]) == -1
    finally:
        loop.close()


def test_evictions_follow_the_mass():
    """From an empty cache: the oracle, given the mass that the attention returned, evicts the same tokens."""
    K, Hkv, L, steps, vocab = 12, 2, 1, 60, 500
    loop = DecodeLoop(n=2, layers=L, batch=1, Hq=4, Hkv=Hkv, K=K, vocab=vocab, seed=3)
    try:
        for t in loop.s.values():
            t.zero_()
        loop.st.cache_len = 0
        pol = oracle_policy(K, "THEOREM", vocab_size=vocab)
        orc = StreamOracle(oracle.Patterns([loop.key_ids], [15.0], [6]), pol, K, L * Hkv)
        for i in range(steps):
            slots = [{int(p): int(r) for p, r in zip(loop.s["pos"][u, :loop.st.cache_len], loop.s["slot"][u, :loop.st.cache_len])}
                     for u in range(L * Hkv)]
            for u in range(L * Hkv):
                slots[u][i] = int(loop.s["next_slot"][u])
            ids = torch.tensor([loop.key_ids[i % 9] if i % 9 < 2 else 100 + i], dtype=torch.int32, device="cuda")
            loop.step(ids, loop._randn(L, 1, 4, 1, 128), loop._randn(L, 1, Hkv, 1, 128), loop._randn(L, 1, Hkv, 1, 128))
            torch.cuda.synchronize()
            mass = loop.mass.view(L * Hkv, K + 1).cpu().numpy().astype(np.float32)
            want = orc.step(int(ids[0]), [{p: mass[u, r] for p, r in slots[u].items()} for u in range(L * Hkv)])
            assert loop.evicted.cpu().tolist() == [int(x) for x in want], i
        assert ta.ta_ctx_poll(loop.ctx) == ta.TA_OK
    finally:
        loop.close()

"""The operators of a decode step over a retained cache, as measurable cases: rotary positions, writing a cache (in fewer
bits) and reading it back, and the attention of new tokens over it.

A case is a plain dict. `path` names the operator; the other fields are its sizes:

  rotate   ta_rotate on the queries and keys of a batch
  cache    ta_cache_append of a batch's keys and values, then ta_cache_read of the same rows
  gather   ta_cache_read of chosen rows of a filled cache (the rows a retention decision keeps)
  attend   ta_attend of `tokens` new tokens per sequence over a filled cache
  step     ta_cache_append of one new token per sequence, then ta_attend over the cache that now holds it, with the
           attention mass that the decode-loop retention step takes

Where `own` is false a pass computes the same from elementary torch operations in 32 bits. Sizes follow the
configurations of this repository (32 query and 8 KV heads of 128 dimensions, 4096 to 131072 tokens, 1 to 64 sequences,
budgets up to 4096), and shards and odd lengths of them. Queries, keys and values are N(0, 1) in bf16.
"""
import math
import random

import torch

own = False

DEV = "cuda:0"
FULL = {"e4m3": 448.0, "int8": 127.0}  # the largest code of a format
TYPES = {"bf16": torch.bfloat16, "e4m3": torch.float8_e4m3fn, "int8": torch.int8}

# ------------------------------------------------------------------------------------------------ the cases


def _rotate(**kw):
    return dict(dict(path="rotate", layers=1, batch=1, n_lo=1, n_hi=1, heads=32, kv=8, d=128, d_rot=128, layout="half",
                     scaling="plain", inverse=False, fused=False, start=0), **kw)


def _cache(**kw):
    return dict(dict(path="cache", layers=1, batch=1, n_lo=1, n_hi=1, start=0, kv=8, d=128, page=16, order="heads",
                     format="bf16", rotary=False), **kw)


def _attend(**kw):
    return dict(dict(path="attend", layers=1, batch=1, n_lo=4096, n_hi=4096, heads=32, kv=8, d=128, page=16, order="heads",
                     format="bf16", tokens=1, causal=True, empty=False, rotary=False), **kw)


def listed():
    return [
        # rotary positions of one new token of 16 sequences deep in their contexts: launch latency
        _rotate(name="rotate_token", batch=16, start=30000),
        # a ragged batch of prompts straight out of a fused projection: strided, neighbouring pairs, half of each head, scaled
        _rotate(name="rotate_ragged", batch=16, n_lo=501, n_hi=8001, d_rot=64, layout="interleaved", scaling="band", fused=True),
        # turning long prompts' keys and queries back (the gradient's direction), positions scaled for 131072 tokens
        _rotate(name="rotate_back_32k", batch=4, n_lo=32768, n_hi=32768, scaling="ramp", inverse=True),
        # one new token of 64 conversations into 8-bit pages, rotated on the way, and read back: launch latency
        _cache(name="cache_token_e4m3", batch=64, start=16000, format="e4m3", rotary=True),
        # a prompt of odd length into whole-number pages that keep all heads of a token together
        _cache(name="cache_prompt_int8", layers=4, n_lo=8111, n_hi=8111, page=64, order="rows", format="int8"),
        # 16 long prompts into 8-bit pages, rotated on the way
        _cache(name="cache_batch_e4m3", layers=2, batch=16, n_lo=32768, n_hi=32768, page=64, format="e4m3", rotary=True),
        # the rows that a budget of 2048 keeps, read out of an 8-bit paged cache of long prompts
        dict(name="gather_2048", path="gather", layers=8, batch=16, n_lo=20000, n_hi=32768, kv=8, d=128, page=16, order="heads",
             format="e4m3", keep=2048),
        # one new token of one 4096-token prompt: the smallest attention call, paid per layer and token
        _attend(name="attend_4k"),
        # one new token of 16 long prompts: throughput serving
        _attend(name="attend_batch_32k", batch=16, n_lo=32768, n_hi=32768, page=64),
        # an agent server's ragged batch over an 8-bit cache, one conversation still empty
        _attend(name="attend_ragged_e4m3", batch=64, n_lo=2048, n_hi=16384, format="e4m3", order="rows", empty=True, rotary=True),
        # four proposed tokens checked at once against very long contexts in whole numbers, a shard's heads
        _attend(name="attend_4_of_131k", batch=4, n_lo=100001, n_hi=131072, heads=16, kv=4, page=64, format="int8", tokens=4),
        # a decode step of the retention loop: all layers, 257 dense rows per head, the new token (queries and keys already
        # rotated) in the row that was freed
        dict(name="step_256", path="step", layers=32, batch=16, heads=32, kv=8, d=128, keep=256),
    ]


MAX_ROWS = 16 * 32768 * 8  # rows of keys (and of values) that a drawn attention or write covers at most


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    path = rng.choices(["rotate", "cache", "gather", "attend", "step"], [3, 3, 1, 5, 1])[0]
    heads, kv = rng.choice([(32, 8), (32, 8), (8, 2), (16, 4), (8, 8), (16, 2), (16, 1), (6, 2), (12, 4)])
    d = rng.choice([128, 128, 128, 64])
    batch = _log_int(rng, 1, 64)
    if path == "step":
        keep = _log_int(rng, 16, 4096)
        layers = max(1, min(_log_int(rng, 1, 32), MAX_ROWS // (batch * kv * (keep + 1))))
        return dict(path=path, layers=layers, batch=batch, heads=heads, kv=kv, d=d, keep=keep)
    layers = rng.choice([1, 1, 1, 2, 4])
    n = _log_int(rng, 1 if path in ("rotate", "cache") else 16, 131072)
    n = max(1, min(n, MAX_ROWS // (batch * layers * kv * (heads // kv if path == "rotate" else 1))))
    lo = n if batch == 1 or rng.random() < 0.4 else max(1, n // 8)
    if path == "rotate":
        layout = rng.choice(["half", "interleaved"])
        return _rotate(layers=layers, batch=batch, n_lo=lo, n_hi=n, heads=heads, kv=kv, d=d,
                       d_rot=rng.choice([d, d, d // 2, d // 4, d - 24]), layout=layout,
                       scaling=rng.choice(["plain", "linear", "base", "ramp", "band"]), inverse=rng.random() < 0.3,
                       fused=rng.random() < 0.5, start=rng.choice([0, 0, 1000, 100001]))
    page, order = rng.choice([1, 16, 16, 48, 64, 128]), rng.choice(["heads", "rows"])
    form = rng.choice(["bf16", "e4m3", "int8"])
    if path == "cache":
        return _cache(layers=layers, batch=batch, n_lo=lo, n_hi=n, start=rng.choice([0, 0, 37, 5000]), kv=kv, d=d, page=page,
                      order=order, format=form, rotary=rng.random() < 0.5)
    if path == "gather":
        return dict(path=path, layers=layers, batch=batch, n_lo=lo, n_hi=n, kv=kv, d=d, page=page, order=order, format=form,
                    keep=_log_int(rng, 1, min(4096, n)))
    return _attend(layers=layers, batch=batch, n_lo=lo, n_hi=n, heads=heads, kv=kv, d=d, page=page, order=order, format=form,
                   tokens=rng.choice([1, 1, 1, 2, 4, 7]), causal=rng.random() < 0.8, empty=batch > 1 and rng.random() < 0.2,
                   rotary=rng.random() < 0.4)


# ------------------------------------------------------------------------------------------------ inputs


def _lengths(case):
    """Tokens of every sequence; a ragged batch's lengths are the same whatever the seed of the inputs."""
    lo, hi, b = case["n_lo"], case["n_hi"], case["batch"]
    rng = random.Random(1000003 * lo + 1009 * hi + b)
    n = [hi if lo == hi else rng.randint(lo, hi) for _ in range(b)]
    if case.get("empty"):
        n[b // 2] = 0
    return n


SCALINGS = {  # kind: (factor, original length, low, high)
    "plain": (1.0, 4096, 0.0, 0.0), "linear": (4.0, 4096, 0.0, 0.0), "base": (4.0, 4096, 0.0, 0.0),
    "ramp": (32.0, 4096, 1.0, 32.0), "band": (8.0, 8192, 1.0, 4.0)}
BASE = 500000.0


def _frequencies(d_rot, scaling):
    """Radians per position of every pair (64 bits), and the factor on the rotated values."""
    factor, original, low, high = SCALINGS[scaling]
    base = BASE * factor ** (d_rot / (d_rot - 2)) if scaling == "base" else BASE
    f = [base ** (-2.0 * i / d_rot) for i in range(d_rot // 2)]
    if scaling == "linear":
        f = [x / factor for x in f]
    if scaling == "ramp":  # whole turns within the original length: many keep their speed, few are slowed down
        def pair_of(turns):
            return d_rot * math.log(original / (turns * 2 * math.pi)) / (2 * math.log(BASE))
        a, b = max(math.floor(pair_of(high)), 0), min(math.ceil(pair_of(low)), d_rot - 1)
        keep = [1 - min(max((i - a) / max(b - a, 0.001), 0.0), 1.0) for i in range(d_rot // 2)]
        return [x / factor * (1 - k) + x * k for x, k in zip(f, keep)], 0.1 * math.log(factor) + 1.0
    if scaling == "band":
        keep = [min(max((original * x / (2 * math.pi) - low) / (high - low), 0.0), 1.0) for x in f]
        f = [x / factor * (1 - k) + x * k for x, k in zip(f, keep)]
    return f, 1.0


def _turns(d_rot, scaling):
    """Turns per position as 64-bit fractions, so that a position's angle is a product modulo 2^64."""
    f, _ = _frequencies(d_rot, scaling)
    whole = [int(x / (2 * math.pi) * 2.0 ** 64) % 2 ** 64 for x in f]
    return torch.tensor([x - 2 ** 64 if x >= 2 ** 63 else x for x in whole], dtype=torch.int64, device=DEV)


def _ints(v, dtype=torch.int32):
    return torch.tensor(v, dtype=dtype, device=DEV)


def _offsets(lens):
    cu = [0]
    for n in lens:
        cu.append(cu[-1] + n)
    return cu


def _randn(gen, *shape):
    return torch.randn(shape, generator=gen, device=DEV, dtype=torch.bfloat16)


def _quantise(x, form):
    """Codes and scales of rows of 32-bit values."""
    top = x.abs().amax(-1, keepdim=True).clamp_min(2.0 ** -100)
    y = x * (FULL[form] / top)
    code = y.round() if form == "int8" else y.clamp(-448.0, 448.0)
    return code.to(TYPES[form]), (top / FULL[form])[..., 0]


def _codes(t):
    """A pool for indexing: 8-bit codes as whole numbers, whatever they stand for."""
    return t.view(torch.int8) if t.element_size() == 1 else t


def _rows_first(case):
    return case.get("order") == "rows"


def _pool(case, gen, pages, filled):
    """Pools [L, pages, kv, page, d] of keys and values with their scales, in the order of the case."""
    L, kv, page, d, form = case["layers"], case["kv"], case["page"], case["d"], case["format"]
    shape = (L, pages, page, kv, d) if _rows_first(case) else (L, pages, kv, page, d)
    turn = (lambda t: t.transpose(2, 3)) if _rows_first(case) else (lambda t: t)
    s = {}
    for name in ("k", "v"):
        if not filled:
            rows = torch.zeros(shape, device=DEV, dtype=torch.bfloat16)
        else:
            rows = _randn(gen, *shape)
        if form == "bf16":
            s[name], s[name + "_scale"] = turn(rows), None
            continue
        code, scale = torch.empty(shape, device=DEV, dtype=TYPES[form]), torch.empty(shape[:-1], device=DEV)
        for l in range(L):
            code[l], scale[l] = _quantise(rows[l].float(), form)
        s[name], s[name + "_scale"] = turn(code), turn(scale)
    return s


def _table(case, gen, rows):
    """A page table for `rows` rows per sequence: pages in no order, what no row needs is -1."""
    need = [-(-r // case["page"]) for r in rows]
    pages = torch.randperm(sum(need) + 3, generator=gen, device=DEV).to(torch.int32)
    table = torch.full((len(rows), max(max(need), 1)), -1, dtype=torch.int32, device=DEV)
    table[torch.arange(table.shape[1], device=DEV) < _ints(need).view(-1, 1)] = pages[:sum(need)]
    return table, sum(need) + 3


def prepare(case, seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    s = {"path": case["path"], "case": case, "gen": gen}
    {"rotate": _prepare_rotate, "cache": _prepare_cache, "gather": _prepare_gather, "attend": _prepare_attend,
     "step": _prepare_step}[case["path"]](case, gen, s)
    del s["gen"]
    s["hands"] = _hands(case, s)
    return s


def _prepare_rotate(case, gen, s):
    L, H, kv, d = case["layers"], case["heads"], case["kv"], case["d"]
    lens = _lengths(case)
    total = sum(lens)
    if case["fused"]:  # one projection's output holds queries, keys and values of a token side by side
        x = _randn(gen, L, total, H + 2 * kv, d)
        q, k = x[:, :, :H], x[:, :, H:H + kv]
    else:
        q, k = _randn(gen, L, total, H, d), _randn(gen, L, total, kv, d)
    s["q"], s["k"] = q.transpose(1, 2), k.transpose(1, 2)  # [L, heads, total, d]
    s["positions"] = torch.cat([torch.arange(n, device=DEV, dtype=torch.int32) + (case["start"] + 17 * b) for b, n in enumerate(lens)])
    s["lens"], s["cu"] = lens, _ints(_offsets(lens))
    s["turns"] = _turns(case["d_rot"], case["scaling"])
    s["q_out"] = torch.empty((L, total, H, d), device=DEV, dtype=torch.bfloat16).transpose(1, 2)
    s["k_out"] = torch.empty((L, total, kv, d), device=DEV, dtype=torch.bfloat16).transpose(1, 2)


def _prepare_cache(case, gen, s):
    L, kv, d = case["layers"], case["kv"], case["d"]
    lens = _lengths(case)
    total, held = sum(lens), [case["start"] + 3 * b for b in range(case["batch"])]
    s["new_k"], s["new_v"] = (_randn(gen, L, total, kv, d).transpose(1, 2) for _ in range(2))
    s["table"], pages = _table(case, gen, [n + h for n, h in zip(lens, held)])
    s.update(_pool(case, gen, pages, False))
    s["lens"], s["cu"], s["held"], s["pages"] = lens, _ints(_offsets(lens)), _ints(held), pages
    s["seq"] = torch.repeat_interleave(torch.arange(case["batch"], device=DEV), _ints(lens, torch.int64))
    row = torch.cat([torch.arange(n, device=DEV, dtype=torch.int32) + h for n, h in zip(lens, held)])
    s["row"] = row
    s["rows"] = row.expand(L, kv, total).contiguous()  # [L][Hkv][total]
    s["turns"] = _turns(d, "plain")
    s["k_out"], s["v_out"] = (torch.empty((L, kv, total, d), device=DEV, dtype=torch.bfloat16) for _ in range(2))


def _prepare_gather(case, gen, s):
    L, B, kv, d, keep = case["layers"], case["batch"], case["kv"], case["d"], case["keep"]
    lens = _lengths(case)
    s["table"], pages = _table(case, gen, lens)
    s.update(_pool(case, gen, pages, True))
    s["lens"], s["held"], s["pages"] = lens, _ints(lens), pages
    # ascending rows of every unit, -1 behind a sequence's last one, as a selection leaves them
    n = _ints(lens, torch.int64).view(1, B, 1, 1)
    at = torch.arange(keep, device=DEV).view(1, 1, 1, keep)
    step = torch.rand((L, B, kv, keep), generator=gen, device=DEV)
    rows = torch.minimum(((at + step) * n / keep).long(), n - 1) if min(lens) >= keep else at.expand(L, B, kv, keep)
    s["rows"] = torch.where(at < n, rows, -1).to(torch.int32).contiguous()
    s["k_out"], s["v_out"] = (torch.empty((L, B, kv, keep, d), device=DEV, dtype=torch.bfloat16) for _ in range(2))


def _prepare_attend(case, gen, s):
    L, B, H, d, T = case["layers"], case["batch"], case["heads"], case["d"], case["tokens"]
    lens = _lengths(case)
    s["table"], pages = _table(case, gen, lens)
    s.update(_pool(case, gen, pages, True))
    s["q"] = _randn(gen, L, B, T, H, d).transpose(2, 3)
    s["lens"], s["held"], s["pages"] = lens, _ints(lens), pages
    s["turns"] = _turns(d, "plain")
    s["out"] = torch.empty((L, B, T, H, d), device=DEV, dtype=torch.bfloat16).transpose(2, 3)
    s["lse"] = torch.empty((L, B, H, T), device=DEV)


def _prepare_step(case, gen, s):
    L, B, H, kv, d, rows = case["layers"], case["batch"], case["heads"], case["kv"], case["d"], case["keep"] + 1
    s["k"], s["v"] = _randn(gen, L, B, kv, rows, d), _randn(gen, L, B, kv, rows, d)
    s["new_k"], s["new_v"] = _randn(gen, L, B, 1, kv, d).transpose(2, 3), _randn(gen, L, B, 1, kv, d).transpose(2, 3)
    s["q"] = _randn(gen, L, B, 1, H, d).transpose(2, 3)
    s["rows"] = torch.randint(0, rows, (L, B, kv, 1), generator=gen, device=DEV, dtype=torch.int32)
    s["out"] = torch.empty((L, B, 1, H, d), device=DEV, dtype=torch.bfloat16).transpose(2, 3)
    s["lse"], s["mass"] = torch.empty((L, B, H, 1), device=DEV), torch.empty((L, B, kv, rows), device=DEV)


# ------------------------------------------------------------------------------------------------ the library's calls

_CONTEXTS = {}  # scratch bytes -> context; a program keeps one, here it is the smallest that suffices


def _phase(ta, d_rot, scaling):
    kinds = {"plain": ta.TA_SCALING_PLAIN, "linear": ta.TA_SCALING_LINEAR, "base": ta.TA_SCALING_BASE, "ramp": ta.TA_SCALING_RAMP,
             "band": ta.TA_SCALING_BAND}
    phase = torch.empty(d_rot // 2, dtype=torch.int64)
    magnitude = ta.ta_rotary_table(d_rot, BASE, kinds[scaling], *SCALINGS[scaling], phase)
    return phase.to(DEV), magnitude


def _hands(case, s):
    """What a program of the library keeps for its calls: the context, and descriptions of its buffers. None in the plain form."""
    if not own:
        return None
    import paper_2604_11288_b200 as ta
    path, h = case["path"], {"ta": ta}
    stream = torch.cuda.current_stream()
    h["stream"] = stream.cuda_stream
    need = 1 << 20
    if path in ("rotate", "cache"):
        lens = s["lens"]
        h["batch"] = ta.make_batch(case["layers"], case["batch"], 0, max(lens), sum(lens), s["cu"])
    if path in ("cache", "gather", "attend"):
        h["cache"] = ta.make_cache(s["k"], s["v"], s["k_scale"], s["v_scale"], table=s["table"], lens=s["held"])
    if path == "gather":
        h["batch"] = ta.make_batch(case["layers"], case["batch"], case["keep"], case["keep"], case["batch"] * case["keep"])
    if path == "step":
        h["batch"] = ta.make_batch(case["layers"], case["batch"], 1, 1, case["batch"])
        h["cache"] = ta.make_cache(s["k"], s["v"], batch=case["batch"], len_uniform=case["keep"] + 1)
    if path in ("attend", "step"):
        h["max_len"] = max(s["lens"] + [1]) if path == "attend" else case["keep"] + 1
        need = max(need, ta.ta_attend_scratch_bytes(h["cache"], case["heads"], case.get("tokens", 1), h["max_len"], path == "step"))
    if path == "rotate":
        layout = {"half": ta.TA_ROTARY_HALF, "interleaved": ta.TA_ROTARY_INTERLEAVED}[case["layout"]]
        phase, magnitude = _phase(ta, case["d_rot"], case["scaling"])
        h["phase"] = phase
        h["rotary"] = ta.make_rotary(phase, case["d_rot"], layout, magnitude, case["inverse"], s["positions"])
    elif case.get("rotary"):
        phase, magnitude = _phase(ta, case["d"], "plain")
        h["phase"] = phase
        h["rotary"] = ta.make_rotary(phase, case["d"], ta.TA_ROTARY_HALF, magnitude, False)
    else:
        h["rotary"] = None
    views = {"rotate": ("q", "k", "q_out", "k_out"), "cache": ("new_k", "new_v", "k_out", "v_out"), "gather": ("k_out", "v_out"),
             "attend": ("q", "out"), "step": ("q", "out", "new_k", "new_v")}[path]
    h.update({n: ta.view(s[n], path in ("rotate", "cache")) for n in views})
    size = 1 << (need - 1).bit_length()
    if size not in _CONTEXTS:
        _CONTEXTS[size] = ta.ta_ctx_create(0, size)
    h["ctx"] = _CONTEXTS[size]
    torch.cuda.synchronize()
    return h


def _run_own(s):
    h, case = s["hands"], s["case"]
    ta, path = h["ta"], s["path"]
    if path == "rotate":
        ta.ta_rotate(h["ctx"], h["batch"], case["heads"], case["kv"], case["d"], h["rotary"], h["q"], h["q_out"], h["k"], h["k_out"],
                     h["stream"])
        return {"q": s["q_out"], "k": s["k_out"]}
    if path == "cache":
        ta.ta_cache_append(h["ctx"], h["cache"], h["batch"], h["rotary"], h["new_k"], h["new_v"], None, h["stream"])
    if path in ("cache", "gather"):
        ta.ta_cache_read(h["ctx"], h["cache"], h["batch"], s["rows"], h["k_out"], h["v_out"], h["stream"])
        return _written(s, s["k_out"], s["v_out"])
    if path == "attend":
        ta.ta_attend(h["ctx"], h["cache"], case["heads"], case["tokens"], 0, h["max_len"], case["causal"], 0.0, h["rotary"], h["q"],
                     h["out"], s["lse"], None, 0, h["stream"])
        return {"out": s["out"], "lse": s["lse"]}
    ta.ta_cache_append(h["ctx"], h["cache"], h["batch"], h["rotary"], h["new_k"], h["new_v"], s["rows"], h["stream"])
    ta.ta_attend(h["ctx"], h["cache"], case["heads"], 1, 0, h["max_len"], True, 0.0, h["rotary"], h["q"], h["out"], s["lse"],
                 s["mass"], case["keep"] + 1, h["stream"])
    return {"out": s["out"], "lse": s["lse"], "mass": s["mass"], "k": s["k"], "v": s["v"]}


def _written(s, k, v):
    r = {"k": k, "v": v}
    if s["path"] == "cache" and s["k_scale"] is not None:
        r.update(k_scale=s["k_scale"], v_scale=s["v_scale"])
    return r


# ------------------------------------------------------------------------------------------------ the plain form


def _cos_sin(positions, turns, magnitude):
    """[..., pairs] of a position's angles: its product with the turns modulo 2^64, the upper half as a fraction of a turn."""
    angle = ((positions.long().unsqueeze(-1) * turns) >> 32).float() * (math.pi / 2.0 ** 31)
    return angle.cos() * magnitude, angle.sin() * magnitude


def _rotated(x, cos, sin, d_rot, layout):
    """Rows x [..., d] in 32 bits with their first d_rot dimensions rotated."""
    head = x[..., :d_rot]
    if layout == "half":
        a, b = head[..., :d_rot // 2], head[..., d_rot // 2:]
        head = torch.cat((a * cos - b * sin, a * sin + b * cos), -1)
    else:
        a, b = head[..., 0::2], head[..., 1::2]
        head = torch.stack((a * cos - b * sin, a * sin + b * cos), -1).flatten(-2)
    return torch.cat((head, x[..., d_rot:]), -1)


def _gathered(s, name, table):
    """Rows [L, B, kv, pages * page, d] of every sequence, in 32 bits."""
    pool, scale = s[name], s[name + "_scale"]
    at = table.clamp_min(0).long()
    x = _codes(pool)[:, at].view(pool.dtype).float()  # [L, B, pages, kv, page, d]
    if scale is not None:
        x = x * scale[:, at].unsqueeze(-1)
    return x.transpose(2, 3).flatten(3, 4)


def _softmax_sums(q, k, v, seen):
    """q [L, B, kv, G, T, d], k and v [L, B, kv, n, d], seen [B, 1, 1, T, n]: output, log-sum-exp and probabilities."""
    sc = torch.einsum("lbhgtd,lbhnd->lbhgtn", q, k) * (1.0 / math.sqrt(q.shape[-1]))
    sc = sc.masked_fill(~seen, -math.inf)
    top = sc.amax(-1, keepdim=True).clamp_min(-1e30)
    e = (sc - top).exp()
    z = e.sum(-1, keepdim=True)
    p = e / z.clamp_min(1e-30)
    out = torch.einsum("lbhgtn,lbhnd->lbhgtd", p, v)
    return out, (top + z.log())[..., 0], p


def run(state):
    if own:
        return _run_own(state)
    s, case = state, state["case"]
    if s["path"] == "rotate":
        cos, sin = _cos_sin(s["positions"], s["turns"], _frequencies(case["d_rot"], case["scaling"])[1])
        sin = -sin if case["inverse"] else sin
        s["q_out"].copy_(_rotated(s["q"].float(), cos, sin, case["d_rot"], case["layout"]))
        s["k_out"].copy_(_rotated(s["k"].float(), cos, sin, case["d_rot"], case["layout"]))
        return {"q": s["q_out"], "k": s["k_out"]}
    if s["path"] == "cache":
        return _run_cache(s, case)
    if s["path"] == "gather":
        return _run_gather(s, case)
    if s["path"] == "attend":
        return _run_attend(s, case)
    return _run_step(s, case)


def _run_cache(s, case):
    page, form = case["page"], case["format"]
    k, v = s["new_k"].float(), s["new_v"].float()  # [L, kv, total, d]
    if case["rotary"]:
        cos, sin = _cos_sin(s["row"], s["turns"], 1.0)
        k = _rotated(k, cos, sin, case["d"], "half")
    at, off = s["table"].long()[s["seq"], s["row"].long() // page], s["row"].long() % page
    for name, x in (("k", k), ("v", v)):  # pool[l, at, h, off]
        code, scale = (x.to(torch.bfloat16), None) if form == "bf16" else _quantise(x, form)
        _codes(s[name]).transpose(2, 3)[:, at, off] = _codes(code).transpose(1, 2)
        if scale is not None:
            s[name + "_scale"].transpose(2, 3)[:, at, off] = scale.transpose(1, 2)
        back = _codes(s[name]).transpose(2, 3)[:, at, off].view(s[name].dtype).float()
        if scale is not None:
            back = back * s[name + "_scale"].transpose(2, 3)[:, at, off].unsqueeze(-1)
        s[name + "_out"].copy_(back.transpose(1, 2))
    return _written(s, s["k_out"], s["v_out"])


def _run_gather(s, case):
    L, B, kv, keep = s["rows"].shape
    rows = s["rows"].long()
    asked = rows.clamp_min(0)
    at = torch.gather(s["table"].long().view(1, B, 1, -1).expand(L, B, kv, -1), 3, asked // case["page"]).clamp_min(0)
    lay, head = torch.arange(L, device=DEV).view(L, 1, 1, 1), torch.arange(kv, device=DEV).view(1, 1, kv, 1)
    for name in ("k", "v"):
        x = _codes(s[name])[lay, at, head, asked % case["page"]].view(s[name].dtype).float()
        if s[name + "_scale"] is not None:
            x = x * s[name + "_scale"][lay, at, head, asked % case["page"]].unsqueeze(-1)
        s[name + "_out"].copy_(x.masked_fill((rows < 0).unsqueeze(-1), 0.0))
    return {"k": s["k_out"], "v": s["v_out"]}


def _seen(case, held, n, T):
    """[B, 1, 1, T, n]: whether query t of a sequence of `held` rows sees row j."""
    last = held.long().view(-1, 1) - (T - 1 - torch.arange(T, device=DEV) if case.get("causal", True) else 0 * torch.arange(T, device=DEV))
    return torch.arange(n, device=DEV).view(1, 1, 1, 1, n) < last.view(-1, 1, 1, T, 1)


def _run_attend(s, case):
    L, B, H, T, d = s["q"].shape
    kv = case["kv"]
    q = s["q"].float()
    if case["rotary"]:  # a query's position is that of the last row it sees in its sequence's order
        cos, sin = _cos_sin(s["held"].view(-1, 1) - (T - torch.arange(T, device=DEV)), s["turns"], 1.0)
        q = _rotated(q, cos.view(B, 1, T, -1), sin.view(B, 1, T, -1), d, "half")
    k, v = _gathered(s, "k", s["table"]), _gathered(s, "v", s["table"])
    out, lse, _ = _softmax_sums(q.view(L, B, kv, H // kv, T, d), k, v, _seen(case, s["held"], k.shape[3], T))
    empty = _seen(case, s["held"], 1, T)[..., 0].logical_not()  # [B, 1, 1, T]
    s["out"].copy_(out.masked_fill(empty.unsqueeze(-1), 0.0).flatten(2, 3))
    s["lse"].copy_(lse.masked_fill(empty, -math.inf).flatten(2, 3))
    return {"out": s["out"], "lse": s["lse"]}


def _run_step(s, case):
    L, B, H, T, d = s["q"].shape
    kv, rows = case["kv"], case["keep"] + 1
    at = s["rows"].long().unsqueeze(-1).expand(L, B, kv, 1, d)
    s["k"].scatter_(3, at, s["new_k"])
    s["v"].scatter_(3, at, s["new_v"])
    q = s["q"].float()
    seen = torch.ones((1, 1, 1, 1, rows), dtype=torch.bool, device=DEV)
    out, lse, p = _softmax_sums(q.view(L, B, kv, H // kv, T, d), s["k"].float(), s["v"].float(), seen)
    s["out"].copy_(out.flatten(2, 3))
    s["lse"].copy_(lse.flatten(2, 3))
    s["mass"].copy_(p.sum((3, 4)))
    return {"out": s["out"], "lse": s["lse"], "mass": s["mass"], "k": s["k"], "v": s["v"]}


# ------------------------------------------------------------------------------------------------ what cannot be done without


def work(case):
    path, d = case["path"], case["d"]
    if path == "rotate":
        elements = case["layers"] * sum(_lengths(case)) * (case["heads"] + case["kv"]) * d
        return {"bytes": 4 * elements, "flops": 3 * elements}
    if path == "step":
        rows = case["layers"] * case["batch"] * case["kv"] * (case["keep"] + 1)
        q = case["layers"] * case["batch"] * case["heads"] * d
        return {"bytes": rows * (4 * d + 4) + 4 * q, "flops": 4 * d * rows * (case["heads"] // case["kv"])}
    held = 2 * d if case["format"] == "bf16" else d + 4  # bytes of a row in the cache
    if path == "gather":
        rows = 2 * case["layers"] * case["kv"] * sum(min(n, case["keep"]) for n in _lengths(case))
        return {"bytes": rows * (held + 2 * d), "flops": rows * d}
    rows = 2 * case["layers"] * case["kv"] * sum(_lengths(case))
    if path == "cache":
        return {"bytes": 2 * rows * (held + 2 * d), "flops": 4 * rows * d}
    q = case["layers"] * case["batch"] * case["heads"] * case["tokens"] * d
    return {"bytes": rows * held + 4 * q, "flops": 2 * rows * d * case["tokens"] * (case["heads"] // case["kv"])}


# ------------------------------------------------------------------------------------------------ the definitions in 64 bits


def _turned64(x, positions, d_rot, layout, scaling, inverse=False):
    """The definition: every pair of coordinates turned by position times frequency. x [..., n, d], positions [..., n]."""
    f, magnitude = _frequencies(d_rot, scaling)
    y = x.clone()
    for i, w in enumerate(f):
        a = positions.double() * w * (-1.0 if inverse else 1.0)
        c, sn = magnitude * torch.cos(a), magnitude * torch.sin(a)
        m, n = (i, i + d_rot // 2) if layout == "half" else (2 * i, 2 * i + 1)
        y[..., m], y[..., n] = x[..., m] * c - x[..., n] * sn, x[..., m] * sn + x[..., n] * c
    return y


def _held64(x, form):
    """What a row of x reads back as from a cache of this format, and its scale."""
    if form == "bf16":
        return x, None
    scale = x.abs().amax(-1, keepdim=True) / FULL[form]
    y = x / scale
    if form == "int8":
        return torch.round(y) * scale, scale[..., 0]
    step = torch.exp2(torch.floor(torch.log2(y.abs().clamp_min(2.0 ** -6))) - 3)  # 3 bits behind the leading one, 2^-9 at least
    return torch.round(y / step) * step * scale, scale[..., 0]


def _rows64(s, name, b, n, page):
    """Rows [L, kv, n, d] that sequence b holds in its pages."""
    j = torch.arange(n, device=DEV)
    at, off = s["table"][b].long()[torch.div(j, page, rounding_mode="floor")], torch.remainder(j, page)
    x = _codes(s[name]).permute(1, 3, 0, 2, 4)[at, off].view(s[name].dtype).float().double()  # [n, L, kv, d]
    if s[name + "_scale"] is not None:
        x = x * s[name + "_scale"].permute(1, 3, 0, 2)[at, off].double().unsqueeze(-1)
    return x.permute(1, 2, 0, 3)


def exact(case, seed):
    s = prepare(case, seed)
    path = case["path"]
    if path == "rotate":
        return {n: _turned64(s[n].double(), s["positions"], case["d_rot"], case["layout"], case["scaling"], case["inverse"])
                for n in ("q", "k")}
    if path == "cache":
        k, v = s["new_k"].double(), s["new_v"].double()
        if case["rotary"]:
            k = _turned64(k, s["row"], case["d"], "half", "plain")
        r, off = {}, s["row"].long() % case["page"]
        at = s["table"].reshape(-1)[s["seq"] * s["table"].shape[1] + torch.div(s["row"].long(), case["page"], rounding_mode="floor")].long()
        for name, x in (("k", k), ("v", v)):
            r[name], scale = _held64(x, case["format"])
            if scale is not None:
                whole = torch.zeros(s[name + "_scale"].shape, dtype=torch.float64, device=DEV)
                whole += s[name + "_scale"].double()  # rows that nobody writes keep what they had
                for h in range(case["kv"]):
                    whole[:, at, h, off] = scale[:, h]
                r[name + "_scale"] = whole
        return r
    if path == "gather":
        r, B = {}, case["batch"]
        for name in ("k", "v"):
            units = []
            for b in range(B):
                x = _rows64(s, name, b, s["lens"][b], case["page"])  # [L, kv, n, d]
                rows = s["rows"][:, b].long()
                y = torch.gather(x, 2, rows.clamp_min(0).unsqueeze(-1).expand(-1, -1, -1, case["d"]))
                units.append(y * (rows >= 0).unsqueeze(-1))
            r[name] = torch.stack(units, 1)
        return r
    L, B, H, T, d = s["q"].shape
    kv, G = case["kv"], H // case["kv"]
    out, lse = torch.zeros((L, B, H, T, d), dtype=torch.float64, device=DEV), torch.full((L, B, H, T), -math.inf, dtype=torch.float64, device=DEV)
    mass = torch.zeros((L, B, kv, case["keep"] + 1), dtype=torch.float64, device=DEV) if path == "step" else None
    if path == "step":
        for l in range(L):
            for b in range(B):
                for h in range(kv):
                    i = int(s["rows"][l, b, h, 0])
                    s["k"][l, b, h, i], s["v"][l, b, h, i] = s["new_k"][l, b, h, 0], s["new_v"][l, b, h, 0]
    for b in range(B):
        n = case["keep"] + 1 if path == "step" else s["lens"][b]
        q = s["q"][:, b].double()
        if path == "step":
            k, v = s["k"][:, b].double(), s["v"][:, b].double()
        else:
            if case["rotary"]:
                q = _turned64(q, n - T + torch.arange(T, device=DEV), d, "half", "plain")
            k, v = (_rows64(s, name, b, n, case["page"]) for name in ("k", "v"))
        for t in range(T):
            last = n - (T - 1 - t) if path == "attend" and case["causal"] else n
            if last <= 0:
                continue
            sc = q[:, :, t].view(L, kv, G, d) @ k[:, :, :last].transpose(-1, -2) / math.sqrt(d)
            lse[:, b, :, t] = torch.logsumexp(sc, -1).flatten(1)
            p = torch.exp(sc - torch.logsumexp(sc, -1, keepdim=True))
            out[:, b, :, t] = (p @ v[:, :, :last]).flatten(1, 2)
            if mass is not None:
                mass[:, b] = p.sum(2)
    if path == "attend":
        return {"out": out, "lse": lse}
    return {"out": out, "lse": lse, "mass": mass, "k": s["k"], "v": s["v"]}

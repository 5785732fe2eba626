"""What stands in front of attention and what a batch shares, as timed calls: the cases that these operators' speed is
measured on, with the operators in plain form.

    rotary        queries and keys turned by their positions, of a prompt or of a batch's new tokens
    norm_rotary   the same behind a norm of every head
    prefix        one generated token of a batch over caches of its own and over caches of prompts that its sequences
                  share

Shapes are those of the workloads in `synth.py` (8 KV heads of dimension 128, 32 or 64 query heads) and the ranges around
them.  All inputs are synthetic and made from the seed alone.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
EPS = 1e-6              # of a norm
TURNS = 4096            # copies of the segment lengths that appending passes take in turn
LOW = -1.0e30           # below every logit
MOST_ELEMENTS = 32768 * 48 * 128        # of a drawn prompt's queries, keys and values
MOST_PAIRS = 8 * 32768 * 64 * 4 + 1     # of a query row and a shared row, in a drawn case
MOST_SHARED = 8 * 32768 + 1             # shared rows of a drawn case
MOST_OWN = 64 * 8 * 1100                # rows of all own caches of a drawn case, spare ones among them


def _turned(kind, dtype, h_q, h_kv, d, tokens, batch=1, place="rows", far=0, layout="half", dims=0, scaling="none", factor=1.0,
            fused=False, name=None):
    """`tokens`: of the longest prompt, the others of a batch down to a sixteenth of it.  `place`: "rows", prompts whose rows
    count from 0; "chunk", a piece of a prompt that begins at position `far`; "spread", a new token of each sequence, at
    positions up to `far`.  `dims`: turned elements of a head, 0 for all of them.  `fused`: queries, keys and values are parts of one tensor's rows."""
    c = dict(kind=kind, dtype=dtype, h_q=h_q, h_kv=h_kv, d=d, tokens=tokens, batch=batch, place=place, far=far, layout=layout,
             dims=dims, scaling=scaling, factor=factor, fused=fused)
    return dict(c, name=name) if name else c


def _prefix(dtype, h_q, h_kv, d, batch, rows, tokens, groups=1, alone=0, kept=0, append=True, name=None):
    """`rows`: a shared cache's rows per head on average, unevenly spread; `groups`: shared caches; `alone`: sequences that
    share none; `kept`: rows per head that a sequence's own prompt left, unevenly spread; `tokens`: rows that every head
    of a sequence has appended, on average."""
    c = dict(kind="prefix", dtype=dtype, h_q=h_q, h_kv=h_kv, d=d, batch=batch, rows=rows, tokens=tokens, groups=groups,
             alone=alone, kept=kept, append=append)
    return dict(c, name=name) if name else c


def listed():
    return [
        # one generated token far into a long context: the latency of the call
        _turned("rotary", "bf16", 32, 8, 128, 1, place="spread", far=131072, scaling="parts", factor=8.0, name="rotary_token"),
        # a long document's queries and keys as the projection leaves them, a schedule for long contexts
        _turned("rotary", "bf16", 32, 8, 128, 32768, scaling="parts", factor=8.0, fused=True, name="rotary_32k"),
        # a served batch of ragged prompts of a small model, half of each head in neighbouring pairs
        _turned("rotary", "fp16", 32, 8, 64, 6011, batch=5, layout="interleaved", dims=32, name="rotary_batch_fp16"),
        # a new token of every sequence of a batch with 64 query heads
        _turned("norm_rotary", "bf16", 64, 8, 128, 64, place="spread", far=65536, name="norm_rotary_step"),
        # a long prompt, the base stretched
        _turned("norm_rotary", "bf16", 32, 8, 128, 16384, scaling="base", factor=4.0, fused=True, name="norm_rotary_16k"),
        # a late piece of a prompt in single precision, an odd part of each head
        _turned("norm_rotary", "fp32", 8, 2, 128, 1021, place="chunk", far=100003, dims=20, scaling="linear", factor=4.0, name="norm_rotary_fp32"),
        # two answers to a short prompt: the latency of the step
        _prefix("bf16", 32, 8, 128, 2, 541, 30, name="prefix_pair"),
        # parallel sampling: sixteen continuations of a compressed document
        _prefix("bf16", 32, 8, 128, 16, 8192, 300, name="prefix_samples"),
        # a served batch behind one long context
        _prefix("bf16", 32, 8, 128, 64, 32768, 500, name="prefix_64"),
        # three documents, questions with compressed prompts of their own, one sequence without a document; 64 query heads
        _prefix("bf16", 64, 8, 128, 8, 16384, 200, groups=3, alone=1, kept=700, name="prefix_documents"),
        # two system prompts of a small model
        _prefix("fp16", 32, 8, 64, 33, 6011, 150, groups=2, name="prefix_fp16"),
        # single precision, attention alone
        _prefix("fp32", 8, 4, 64, 5, 1500, 70, append=False, name="prefix_fp32"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["rotary", "norm_rotary", "prefix", "prefix"])
    h_kv, g, d = rng.choice([2, 4, 8, 8]), rng.choice([1, 2, 4, 4, 8]), rng.choice([64, 128, 128])
    dtype = rng.choice(["bf16", "bf16", "fp16", "fp32"])
    if kind != "prefix":
        place = rng.choice(["rows", "rows", "chunk", "spread"])
        batch = rng.choice([1, 1, 2, 3, 5, 8]) if place == "rows" else 1
        tokens = _log_int(rng, 1, 64) if place == "spread" else _log_int(rng, 2, 32768)
        while batch * tokens * (g + 2) * h_kv * d * (2 if dtype == "fp32" else 1) > MOST_ELEMENTS:
            tokens = tokens * 7 // 8
        return _turned(kind, dtype, g * h_kv, h_kv, d, tokens, batch, place, 0 if place == "rows" else _log_int(rng, 64, 1 << 20),
                       rng.choice(["half", "half", "interleaved"]), rng.choice([0, 0, d // 2, d // 4, 2 * rng.randint(1, d // 2)]),
                       *rng.choice([("none", 1.0), ("linear", 4.0), ("base", 8.0), ("parts", 8.0), ("parts", 32.0)]), rng.random() < 0.5)
    batch = _log_int(rng, 1, 64)
    groups, alone = rng.choice([1, 1, 2, 3]), rng.choice([0, 0, 1])
    groups = min(groups, batch)
    rows, kept, tokens = _log_int(rng, 1, 32768), rng.choice([0, 0, _log_int(rng, 8, 1024)]), _log_int(rng, 1, 1024)
    while rows > 1 and (g * h_kv * batch * rows > MOST_PAIRS or groups * h_kv * rows > MOST_SHARED):
        rows = rows * 7 // 8
    while batch * h_kv * (2 * tokens + 65 + 2 * kept) > MOST_OWN and max(tokens, kept) > 1:
        tokens, kept = max(1, tokens * 7 // 8), kept * 7 // 8
    return _prefix(dtype, g * h_kv, h_kv, d, batch, rows, tokens, groups, min(alone, batch - 1), kept, rng.random() < 0.7)


# ---- what a case stands for, in numbers --------------------------------------------------------------------------
def _prompt_lengths(case):
    """Tokens of each prompt: the longest first, the others spread below it."""
    n, batch = case["tokens"], case["batch"]
    return [n] + [max(2, n // 16 + (n - n // 16) * (batch - i) // (batch + 1) - 7 * i) for i in range(1, batch)]


def _schedule(case):
    """Arguments of the frequencies: the base, how it is scaled, and by how much the turned elements are magnified."""
    long = case["scaling"] == "parts"
    return dict(base=500000.0 if long else 10000.0, scaling=case["scaling"], factor=case["factor"], original_len=8192, low=1.0, high=4.0,
                magnitude=1.0 + 0.1 * math.log(case["factor"]) if long else 1.0)


def _of(case):
    """The shared cache of each sequence, -1 for none; the first ones have the most."""
    u = np.random.Generator(np.random.PCG64(60_000 + case["batch"])).uniform(size=case["batch"])
    of = np.minimum((case["groups"] * u ** 2).astype(int), case["groups"] - 1)
    of[case["batch"] - case["alone"]:] = -1
    return of.tolist()


def _uneven(rng, rows, h, many):
    """Rows of each of many*h segments, as adaptive budgets spread them over the heads."""
    out = []
    for f in rng.uniform(0.5, 1.5, size=many) if many > 1 else [1.0]:
        wgt = np.exp(rng.standard_normal(h))
        out += [max(1, int(v)) for v in rows * f * h * wgt / wgt.sum()]
    return out


def _lengths(case):
    """Rows of the shared segments; rows kept of each own segment; rows held of each own segment.  They go by the case alone."""
    rng = np.random.Generator(np.random.PCG64(61_000 + case["rows"]))
    h, batch = case["h_kv"], case["batch"]
    shared = _uneven(rng, case["rows"], h, case["groups"])
    kept = _uneven(rng, case["kept"], h, batch) if case["kept"] else [1] * (batch * h)
    tokens = [case["tokens"]] + [int(v) for v in rng.uniform(0, 2 * case["tokens"], size=batch - 1)]
    held = [(kept[b * h + c] if case["kept"] else 0) + tokens[b] for b in range(batch) for c in range(h)]
    return shared, kept, held


def _headroom(case):
    return 2 * case["tokens"] + 64


def _int(x, dtype=torch.int32):
    return torch.as_tensor(np.asarray(x), dtype=dtype, device="cuda")


def _starts(lens, headroom):
    cu = np.concatenate([[0], np.cumsum(lens)])
    return cu, cu[:-1] + headroom * np.arange(len(lens))


def _frequencies(m, base, scaling, factor, original_len, low, high, magnitude):
    """Radians a position, of m/2 pairs."""
    if scaling == "base" and m > 2:
        base = base * factor ** (m / (m - 2))
    f = base ** (-torch.arange(0, m, 2, dtype=torch.float64) / m)
    if scaling == "linear":
        f = f / factor
    elif scaling == "parts":
        whole = ((original_len * f / (2 * math.pi) - low) / (high - low)).clamp(0.0, 1.0)
        f = f * (whole + (1 - whole) / factor)
    return f


def _cache_layer(case, lens, batch):
    import paper_2407_11550_amd as adakv
    h = case["h_kv"]
    return adakv.Layer(DTYPES[case["dtype"]], case["h_q"], h, case["d"], 1, 7, 0.2, [max(lens[b * h:(b + 1) * h]) for b in range(batch)],
                       [sum(lens[b * h:(b + 1) * h]) for b in range(batch)])


def _prepare_turned(case, randn):
    dt, h_q, h, d = DTYPES[case["dtype"]], case["h_q"], case["h_kv"], case["d"]
    lens = _prompt_lengths(case)
    rows = sum(lens)
    s = dict(case=case, freq=_frequencies(case["dims"] or d, **_schedule(case)).cuda())
    if case["fused"]:
        x = randn(rows, (h_q + 2 * h) * d, by=2.0).to(dt)
        s["q"], s["k"] = x[:, :h_q * d].view(rows, h_q, d), x[:, h_q * d:(h_q + h) * d].view(rows, h, d)
    else:
        s["q"], s["k"] = randn(rows, h_q, d, by=2.0).to(dt), randn(rows, h, d, by=2.0).to(dt)
    if case["place"] == "rows":
        s["positions"] = None
        s["at"] = _int(np.concatenate([np.arange(n) for n in lens]))
    else:
        rng = np.random.Generator(np.random.PCG64(62_000 + case["tokens"]))
        s["positions"] = s["at"] = _int(case["far"] + np.arange(rows) if case["place"] == "chunk" else rng.integers(0, case["far"], size=rows))
    s["q_out"], s["k_out"] = torch.zeros((rows, h_q, d), dtype=dt, device="cuda"), torch.zeros((rows, h, d), dtype=dt, device="cuda")
    if case["kind"] == "norm_rotary":
        s["q_weight"], s["k_weight"] = (1.0 + randn(d, by=0.2)).to(dt), (1.0 + randn(d, by=0.2)).to(dt)
    if own:
        import paper_2407_11550_amd as adakv
        s["layer"] = adakv.Layer(dt, h_q, h, d, 1, 7, 0.2, [max(1, n - 1) for n in lens], [h for _ in lens])
        s["rotation"] = adakv.Rotary(case["dims"] or d, layout=case["layout"], device="cuda", **_schedule(case))
    return s


def _prepare_prefix(case, randn):
    dt, h_q, h, d, batch = DTYPES[case["dtype"]], case["h_q"], case["h_kv"], case["d"], case["batch"]
    shared, kept, held = _lengths(case)
    headroom, of = _headroom(case), _of(case)
    cu, start = _starts(kept, headroom)
    p_cu, p_start = _starts(shared, 0)
    s = dict(case=case, headroom=headroom, cu=_int(cu), start=_int(start, torch.int64), p_cu=_int(p_cu), p_start=_int(p_start, torch.int64),
             p_len=_int(shared), longest=max(held) + 1, p_longest=max(shared), capacity=_int(np.asarray(kept) + headroom, torch.int64))
    # which sequences look at a shared cache, one behind the other, and which of these places are filled
    members = [[b for b in range(batch) if of[b] == p] for p in range(case["groups"])]
    most = max(len(m) for m in members)
    s["members"] = _int([m + [0] * (most - len(m)) for m in members], torch.int64)
    s["filled"] = _int([[i < len(m) for i in range(most)] for m in members], torch.bool)
    rows = int(cu[-1]) + batch * h * headroom
    at = _int(np.concatenate([np.arange(n) + start[i] for i, n in enumerate(held)]), torch.int64)
    for x in "KV":
        s[x + "_cache"] = torch.zeros((rows, d), dtype=dt, device="cuda")
        s[x + "_cache"][at] = randn(len(at), d).to(dt)
        s["p_" + x] = randn(int(p_cu[-1]), d).to(dt)
    s["q"] = randn(batch, h_q, d, by=2.0).to(dt)
    s["k"], s["v"] = randn(batch, h, d).to(dt), randn(batch, h, d).to(dt)
    lens = _int(held)
    s["turns"], s["turn"] = list(lens.repeat(TURNS, 1).unbind(0)) if case["append"] else [lens], 0
    s["overflow"] = torch.zeros(1, dtype=torch.int32, device="cuda")
    s["out"], s["lse"] = torch.zeros((batch, h_q, d), device="cuda"), torch.zeros((batch, h_q), device="cuda")
    if own:
        import paper_2407_11550_amd as adakv
        s["layer"] = _cache_layer(case, kept, batch)
        s["prefix"] = adakv.Prefix(_cache_layer(case, shared, case["groups"]), s["p_cu"], 0, s["p_K"], s["p_V"], s["p_len"], of)
        s["ws"] = torch.zeros(adakv.prefix_workspace_bytes(s["layer"], headroom, s["prefix"]), dtype=torch.uint8, device="cuda")
    return s


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(80_000 + seed)

    def randn(*shape, by=1.0):
        return torch.randn(shape, generator=gen, device="cuda") * by

    return (_prepare_prefix if case["kind"] == "prefix" else _prepare_turned)(case, randn)


# ---- the operators, plain ----------------------------------------------------------------------------------------
def _turn(s, x, cos, sin, weight):
    case, y = s["case"], x.float()
    if weight is not None:
        y = y * torch.rsqrt((y * y).mean(dim=-1, keepdim=True) + EPS) * weight.float()
    m = case["dims"] or case["d"]
    if case["layout"] == "half":
        a, b = y[..., :m // 2], y[..., m // 2:m]
        turned = torch.cat([a * cos - b * sin, b * cos + a * sin], dim=-1)
    else:
        a, b = y[..., 0:m:2], y[..., 1:m:2]
        turned = torch.stack([a * cos - b * sin, b * cos + a * sin], dim=-1).flatten(-2)
    return torch.cat([turned, y[..., m:]], dim=-1).to(x.dtype)


def _plain_turned(s):
    angle = s["at"].double()[:, None] * s["freq"]
    by = _schedule(s["case"])["magnitude"]
    cos, sin = (torch.cos(angle) * by).float()[:, None], (torch.sin(angle) * by).float()[:, None]
    s["q_out"].copy_(_turn(s, s["q"], cos, sin, s.get("q_weight")))
    s["k_out"].copy_(_turn(s, s["k"], cos, sin, s.get("k_weight")))


def _sums(q, K, V, seen):
    """q [S, m, d] over rows [S, T, d] of which `seen` [S, T] count: the largest logit, the sum of exp below it, the sum of
    such weights times values."""
    x = (torch.matmul(q, K.transpose(1, 2)) / math.sqrt(q.shape[-1])).masked_fill(~seen[:, None], -math.inf)
    top = x.amax(dim=-1, keepdim=True).clamp(min=LOW)
    x = torch.exp(x - top)
    return top, x.sum(dim=-1, keepdim=True), torch.matmul(x, V.masked_fill(~seen[..., None], 0.0))


def _rows(cache, start, lens, longest):
    """Segments of a cache as [segments, longest, d] in 32 bits, and which rows are theirs."""
    t = torch.arange(longest, device="cuda")
    at = (start[:, None] + t).clamp(max=len(cache) - 1)
    return cache[at.reshape(-1)].view(len(start), longest, -1).float(), t < lens[:, None]


def _plain_prefix(s, lens):
    case = s["case"]
    h, d, batch, groups = case["h_kv"], case["d"], case["batch"], case["groups"]
    g, S = case["h_q"] // h, batch * h
    held = lens.long()
    if case["append"]:
        room = held < s["capacity"]
        at = (s["start"] + held).clamp(max=len(s["K_cache"]) - 1)
        for x, new in (("K_cache", s["k"]), ("V_cache", s["v"])):
            s[x][at] = torch.where(room[:, None], new.view(S, d), s[x][at])
        held = held + room
        s["overflow"] |= (~room).any()
        lens.copy_(held)
    q = s["q"].float().view(batch, h, g, d)
    K, seen = _rows(s["K_cache"], s["start"], held, s["longest"])
    V, _ = _rows(s["V_cache"], s["start"], held, s["longest"])
    top, total, acc = (x.view(batch, h, g, -1) for x in _sums(q.view(S, g, d), K, V, seen))
    del K, V, seen
    # the queries of all that share a cache, side by side
    K, seen = _rows(s["p_K"], s["p_start"], s["p_len"], s["p_longest"])
    V, _ = _rows(s["p_V"], s["p_start"], s["p_len"], s["p_longest"])
    many = s["members"].shape[1]
    mine = q[s["members"]].transpose(1, 2).reshape(groups * h, many * g, d)
    parts = [x.view(groups, h, many, g, -1).transpose(1, 2)[s["filled"]] for x in _sums(mine, K, V, seen)]
    who = s["members"][s["filled"]]
    p_top, p_total, p_acc = torch.full_like(top, LOW), torch.zeros_like(total), torch.zeros_like(acc)
    p_top[who], p_total[who], p_acc[who] = parts
    most = torch.maximum(top, p_top)
    a, b = torch.exp(top - most), torch.exp(p_top - most)
    total = total * a + p_total * b
    some = total > 0
    s["out"].copy_(torch.where(some, (acc * a + p_acc * b) / total, 0.0).view(batch, h * g, d))
    s["lse"].copy_(torch.where(some, most + torch.log(total), -math.inf).view(batch, h * g))


def _own_turned(s):
    import paper_2407_11550_amd as adakv
    if s["case"]["kind"] == "rotary":
        adakv.rotary(s["layer"], s["rotation"], s["q"], s["k"], positions=s["positions"], q_out=s["q_out"], k_out=s["k_out"])
    else:
        adakv.norm_rotary(s["layer"], s["rotation"], s["q"], s["k"], s["q_weight"], s["k_weight"], EPS, positions=s["positions"],
                          q_out=s["q_out"], k_out=s["k_out"])


def _own_prefix(s, lens):
    import paper_2407_11550_amd as adakv
    if s["case"]["append"]:
        adakv.decode_prefix_step(s["layer"], s["q"], s["k"], s["v"], s["cu"], s["headroom"], s["K_cache"], s["V_cache"], lens, s["prefix"],
                                 overflow=s["overflow"], out=s["out"], lse=s["lse"], ws=s["ws"])
    else:
        adakv.decode_prefix_attn(s["layer"], s["q"], s["cu"], s["headroom"], s["K_cache"], s["V_cache"], lens, s["prefix"],
                                 out=s["out"], lse=s["lse"], ws=s["ws"])


def run(s):
    if s["case"]["kind"] != "prefix":
        (_own_turned if own else _plain_turned)(s)
        return dict(q=s["q_out"], k=s["k_out"])
    lens = s["turns"][s["turn"]]
    s["turn"] = (s["turn"] + 1) % len(s["turns"])
    (_own_prefix if own else _plain_prefix)(s, lens)
    if not s["case"]["append"]:
        return dict(out=s["out"], lse=s["lse"])
    return dict(out=s["out"], lse=s["lse"], K_cache=s["K_cache"], V_cache=s["V_cache"], seg_len=lens, overflow=s["overflow"])


def work(case):
    e = 4 if case["dtype"] == "fp32" else 2
    h_q, h, d = case["h_q"], case["h_kv"], case["d"]
    if case["kind"] != "prefix":
        rows, m, norm = sum(_prompt_lengths(case)), case["dims"] or d, case["kind"] == "norm_rotary"
        return dict(bytes=2 * rows * (h_q + h) * d * e + (0 if case["place"] == "rows" else 4 * rows) + 4 * m + (2 * d * e if norm else 0),
                    flops=rows * (h_q + h) * (3 * m + (4 * d if norm else 0)))
    shared, _, held = _lengths(case)
    of, g, S, new = _of(case), h_q // h, len(held), int(case["append"])
    pairs = sum(sum(shared[p * h:(p + 1) * h]) for p in of if p >= 0) + sum(held) + S * new
    used = sum(sum(shared[p * h:(p + 1) * h]) for p in set(of) if p >= 0)
    io = case["batch"] * h_q * (d * e + 4 * d + 4) + S * (2 * d * e * 2 + 4) * new + 8 * S
    return dict(bytes=2 * d * e * (used + sum(held)) + io, flops=4 * g * d * pairs)


# ---- the definitions, in 64 bits ---------------------------------------------------------------------------------
def _exact_turned(s):
    case, spec = s["case"], _schedule(s["case"])
    m = case["dims"] or case["d"]
    pairs = m // 2
    base = spec["base"] * (case["factor"] ** (m / (m - 2.0)) if case["scaling"] == "base" and m > 2 else 1.0)
    freq = []
    for i in range(pairs):
        f = math.exp(-2.0 * i / m * math.log(base))
        if case["scaling"] == "linear":
            f /= case["factor"]
        if case["scaling"] == "parts":
            turns = spec["original_len"] * f / math.tau
            share = min(1.0, max(0.0, (turns - spec["low"]) / (spec["high"] - spec["low"])))
            f = share * f + (1.0 - share) * f / case["factor"]
        freq.append(f)
    angle = torch.outer(s["at"].double(), torch.tensor(freq, dtype=torch.float64, device="cuda"))
    spin = torch.polar(torch.full_like(angle, spec["magnitude"]), angle)[:, None, :]
    out = {}
    for name in "qk":
        x = s[name].double()
        if case["kind"] == "norm_rotary":
            x = x / torch.sqrt(torch.mean(x.square(), dim=2, keepdim=True) + EPS) * s[name + "_weight"].double()
        y = x.clone()
        if case["layout"] == "half":
            z = torch.complex(x[:, :, :pairs].contiguous(), x[:, :, pairs:m].contiguous()) * spin
            y[:, :, :pairs], y[:, :, pairs:m] = z.real, z.imag
        else:
            z = torch.view_as_complex(x[:, :, :m].reshape(*x.shape[:2], pairs, 2).contiguous()) * spin
            y[:, :, :m] = torch.view_as_real(z).reshape(*x.shape[:2], m)
        out[name] = y
    return out


def _exact_prefix(s):
    case = s["case"]
    h, g, of = case["h_kv"], case["h_q"] // case["h_kv"], _of(case)
    shared, kept, held = _lengths(case)
    cu, start = _starts(kept, s["headroom"])
    p_cu, _ = _starts(shared, 0)
    K, V = s["K_cache"].double(), s["V_cache"].double()
    if case["append"]:
        for i, n in enumerate(held):
            K[start[i] + n], V[start[i] + n] = s["k"][i // h, i % h].double(), s["v"][i // h, i % h].double()
        held = [n + 1 for n in held]
    out = torch.zeros(s["out"].shape, dtype=torch.float64, device="cuda")
    lse = torch.zeros(s["lse"].shape, dtype=torch.float64, device="cuda")
    for c in range(h):
        theirs = [tuple(s["p_" + x][p_cu[p * h + c]:p_cu[p * h + c + 1]].double() for x in "KV") for p in range(case["groups"])]
        for b in range(case["batch"]):
            i = b * h + c
            keys, values = K[start[i]:start[i] + held[i]], V[start[i]:start[i] + held[i]]
            if of[b] >= 0:
                keys, values = torch.cat([theirs[of[b]][0], keys]), torch.cat([theirs[of[b]][1], values])
            heads = slice(c * g, (c + 1) * g)
            if len(keys) == 0:
                lse[b, heads] = -math.inf
                continue
            logit = (keys @ s["q"][b, heads].double().T.contiguous()).T / math.sqrt(case["d"])
            out[b, heads], lse[b, heads] = torch.softmax(logit, dim=1) @ values, torch.logsumexp(logit, dim=1)
    if not case["append"]:
        return dict(out=out, lse=lse)
    return dict(out=out, lse=lse, K_cache=K, V_cache=V, seg_len=None, overflow=None)


def exact(case, seed):
    s = prepare(case, seed)
    return _exact_prefix(s) if case["kind"] == "prefix" else _exact_turned(s)

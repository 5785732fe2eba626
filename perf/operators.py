"""What surrounds a compressed cache when it is served, as timed calls: the cases that these operators' speed is
measured on, with the operators in plain form.

    prompt        causal attention over a prompt, limited to a window and a few first tokens, with the
                  log-sum-exp of the last rows as the scoring call takes it
    window_step   one generated token over a cache of which only a window and the first rows are looked at
    q8_build      the retained rows into a cache of 8-bit values with a scale per 32 rows of a head
    q8_step       one generated token over such a cache: append and attention
    move          sequences of a cache forked, dropped and set up with other head-room

Shapes are those of the workloads in `synth.py` (8 KV heads of dimension 128, 32 or 64 query heads, window rows 32 or
64) and the ranges around them.  All inputs are synthetic and made from the seed alone.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
F8 = torch.float8_e4m3fn
BLOCK = 32              # rows that share a scale
TOP = 448.0             # the largest e4m3 value
LOW_K, HIGH_K = -60, 100    # exponents of a scale
TURNS = 4096            # copies of the segment lengths that decode passes take in turn
MOST_ROWS = 1 << 20     # cache rows of a drawn case
MOST_LOGITS = 32 * 16384 * 8192 + 1


def _prompt(dtype, h_q, h_kv, d, n, batch, window, sinks, name=None):
    """`n`: tokens of the longest prompt, the others of a batch down to a sixteenth of it; window 0: all tokens."""
    c = dict(kind="prompt", dtype=dtype, h_q=h_q, h_kv=h_kv, d=d, n=n, batch=batch, window=window, sinks=sinks)
    return dict(c, name=name) if name else c


def _cache(kind, dtype, h_q, h_kv, d, batch, rows, headroom=256, window=0, sinks=0, picks="", new_headroom=0, q8=False, n=0, name=None):
    """`rows`: rows per head on average, unevenly spread; `picks`: source sequences of the moved cache, as text."""
    c = dict(kind=kind, dtype=dtype, h_q=h_q, h_kv=h_kv, d=d, batch=batch, rows=rows, headroom=headroom, window=window,
             sinks=sinks, picks=picks, new_headroom=new_headroom, q8=q8, n=n)
    return dict(c, name=name) if name else c


def listed():
    return [
        # a chat turn: a short prompt, all of it visible; the latency of the call
        _prompt("bf16", 32, 8, 128, 541, 1, 0, 0, name="prompt_short"),
        # a long document through a layer with a sliding window and four sinks
        _prompt("bf16", 32, 8, 128, 32768, 1, 4096, 4, name="prompt_32k_window"),
        # the whole prompt visible, at the lengths whose caches get compressed
        _prompt("bf16", 32, 8, 128, 16384, 1, 0, 0, name="prompt_16k"),
        # a served batch of ragged prompts of a small model
        _prompt("fp16", 32, 8, 64, 6011, 5, 1000, 4, name="prompt_batch_fp16"),
        # one token through a sliding-window layer that keeps all rows
        _cache("window_step", "bf16", 32, 8, 128, 8, 20000, window=4096, sinks=4, name="window_step_batch"),
        # the same for one sequence in single precision: the latency of the step
        _cache("window_step", "fp32", 8, 8, 64, 1, 3001, window=509, sinks=1, name="window_step_fp32"),
        # the caches of a prefilled batch at the paper's budgets, into 8 bits
        _cache("q8_build", "bf16", 32, 8, 128, 8, 1500, n=30011, name="q8_build_batch"),
        # one short sequence in single precision
        _cache("q8_build", "fp32", 8, 4, 64, 1, 517, n=4099, name="q8_build_fp32"),
        # one token for one short sequence of a small model: the latency of the step
        _cache("q8_step", "fp16", 32, 8, 64, 1, 512, name="q8_step_small"),
        # one token for a batch at long budgets, 64 query heads
        _cache("q8_step", "bf16", 64, 8, 128, 8, 8192, name="q8_step_64heads"),
        # parallel sampling: one prompt's cache for eight continuations
        _cache("move", "bf16", 32, 8, 128, 2, 4096, headroom=0, picks="0 0 0 0 0 0 0 1", new_headroom=256, name="move_fork"),
        # finished sequences leave an 8-bit batch, the others get room again
        _cache("move", "bf16", 32, 8, 128, 8, 1500, picks="6 0 3 1 4", new_headroom=512, q8=True, name="move_compact_q8"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["prompt", "prompt", "prompt", "window_step", "window_step", "q8_build", "q8_step", "q8_step", "move"])
    h_kv, g, d = rng.choice([2, 4, 8, 8]), rng.choice([1, 2, 4, 4, 8]), rng.choice([64, 128, 128])
    dtype = rng.choice(["bf16", "bf16", "fp16", "fp32"])
    batch = rng.choice([1, 1, 2, 3, 5, 8])
    if kind == "prompt":
        window = rng.choice([0, 0, _log_int(rng, 1, 8192), _log_int(rng, 100, 8192)])
        sinks = rng.choice([0, 1, 4, 4, 70])
        n = _log_int(rng, 2, 16384 if dtype != "fp32" else 4096)
        while batch * g * h_kv * n * min(n, 2 * (window or n)) > MOST_LOGITS:
            n = n * 7 // 8
        return _prompt(dtype, g * h_kv, h_kv, d, n, batch, window, sinks)
    rows = _log_int(rng, 8, min(32768, MOST_ROWS // (batch * h_kv)))
    headroom = rng.choice([32, 100, 256])
    if kind == "window_step":
        return _cache(kind, dtype, g * h_kv, h_kv, d, batch, rows, headroom, _log_int(rng, 1, 8192), rng.choice([0, 1, 4, 4, 70]))
    if kind == "q8_build":
        rows = min(rows, 8192)
        return _cache(kind, dtype, g * h_kv, h_kv, d, batch, rows, headroom, n=4 * rows + _log_int(rng, 1, 8192))
    if kind == "q8_step":
        return _cache(kind, dtype, g * h_kv, h_kv, d, batch, rows, headroom)
    many = rng.choice([1, 2, 5, 8])
    rows = min(rows, max(8, MOST_ROWS // (many * 2 * h_kv)))
    return _cache(kind, dtype, g * h_kv, h_kv, d, batch, rows, headroom, picks=" ".join(str(rng.randrange(batch)) for _ in range(many)),
                  new_headroom=rng.choice([0, 33, 300]) + headroom, q8=rng.random() < 0.5)


# ---- what a case stands for, in numbers --------------------------------------------------------------------------
W = 32                  # observation window of the layers


def _prompt_lengths(case):
    """Tokens of each prompt: the longest first, the others spread below it."""
    n, batch = case["n"], case["batch"]
    return [n] + [max(2, n // 16 + (n - n // 16) * (batch - i) // (batch + 1) - 7 * i) for i in range(1, batch)]


def _kept(case):
    """Rows of each segment [batch*h_kv], which go by the case alone: per sequence a share of the average, spread over its heads as adaptive
    budgets are; a window layer's heads all hold the same."""
    rng = np.random.Generator(np.random.PCG64(50_000 + case["rows"]))
    rows, h, batch = case["rows"], case["h_kv"], case["batch"]
    per = [rows] + [max(2, int(rows * f)) for f in rng.uniform(0.5, 1.5, size=batch - 1)]
    if case["kind"] == "window_step":
        return [v for v in per for _ in range(h)]
    most = case["n"] or 1 << 30
    out = []
    for v in per:
        wgt = np.exp(rng.standard_normal(h))
        out += [int(x) for x in np.clip(np.floor(v * h * wgt / wgt.sum()), 2, most)]
    return out


def _row_window(case):
    """Window rows of the layer, which every head holds."""
    return 2 if case["kind"] != "prompt" else min(W, min(_prompt_lengths(case)) - 1)


def _layer(case, lens):
    """The framework's description of the layer: `lens` are a prompt's tokens, or the rows of a cache's segments."""
    import paper_2407_11550_amd as adakv
    h, w = case["h_kv"], _row_window(case)
    if case["kind"] == "prompt":
        n, B = [v - w for v in lens], [w * h for _ in lens]
    else:
        n = [case["n"] or max(lens[b * h:(b + 1) * h]) for b in range(case["batch"])]
        B = [sum(lens[b * h:(b + 1) * h]) for b in range(case["batch"])]
    return adakv.Layer(DTYPES[case["dtype"]], case["h_q"], h, case["d"], w, 7, 0.2, n, B)


# ---- 8-bit values, plain -----------------------------------------------------------------------------------------
def _pow2(k):
    return ((k.to(torch.int32) + 127) << 23).view(torch.float32)


def _exponent(m):
    """The smallest k with m <= 448 * 2^k, within the limits of a scale."""
    f, e = torch.frexp(m)
    k = torch.where(f <= 0.875, e - 9, e - 8)
    return torch.where(m > 0, k, torch.full_like(k, LOW_K)).clamp(LOW_K, HIGH_K)


def _exponent_of(scale):
    return (scale.view(torch.int32) >> 23) - 127


def _round8(x):
    return torch.where(torch.isfinite(x), x.clamp(-TOP, TOP), torch.full_like(x, math.nan)).to(F8)


def _magnitude(x):
    return torch.where(torch.isfinite(x), x.abs(), torch.zeros_like(x)).amax(dim=-1)


def _quantise(rows, block, blocks):
    """fp32 rows [R, d] of blocks `block` [R] -> codes [R, d], scales [blocks] (0 where a block has no rows)."""
    m = torch.full((blocks,), -1.0, device=rows.device).scatter_reduce(0, block, _magnitude(rows), "amax")
    k = _exponent(m.clamp(min=0.0))
    return _round8(rows * _pow2(-k)[block][:, None]), torch.where(m >= 0, _pow2(k), torch.zeros_like(m))


def _layout(lens, headroom):
    """Where things are: first rows and capacities of the segments, rows and scale blocks in all."""
    cu = np.concatenate([[0], np.cumsum(lens)])
    start = cu[:-1] + headroom * np.arange(len(lens))
    rows = int(cu[-1]) + len(lens) * headroom
    return cu, start, rows, rows // BLOCK + len(lens)


def _int(x, dtype=torch.int32):
    return torch.as_tensor(np.asarray(x), dtype=dtype, device="cuda")


def _rows_of(lens, headroom):
    """Held rows, segment after segment: their place in the cache, their segment, their place in it, their scale."""
    lens = np.asarray(lens)
    cu, start, _, _ = _layout(lens, headroom)
    seg = np.repeat(np.arange(len(lens)), lens)
    t = np.arange(int(cu[-1])) - cu[:-1][seg]
    return start[seg] + t, seg, t, start[seg] // BLOCK + seg + t // BLOCK


def prepare(case, seed):
    dt, d, h, batch = DTYPES[case["dtype"]], case["d"], case["h_kv"], case["batch"]
    gen = torch.Generator(device="cuda")
    gen.manual_seed(70_000 + seed)

    def randn(*shape, by=1.0):
        return torch.randn(shape, generator=gen, device="cuda") * by

    def empty(*shape, dtype=dt):
        return torch.zeros(shape, dtype=dtype, device="cuda")

    s = dict(case=case)
    if case["kind"] == "prompt":
        lens = _prompt_lengths(case)
        s["lens"], tokens, w = lens, sum(lens), _row_window(case)
        s["q"] = randn(tokens, case["h_q"], d, by=1.5).to(dt)
        s["K"], s["V"] = randn(tokens, h, d).to(dt), randn(tokens, h, d).to(dt)
        s["out"], s["row_lse"] = empty(tokens, case["h_q"], d), empty(batch, case["h_q"], w, dtype=torch.float32)
        s["layer"] = _layer(case, lens) if own else None
        return s
    lens = _kept(case)
    headroom = case["headroom"]
    cu, start, rows, blocks = _layout(lens, headroom)
    s["lens"], s["cu"], s["start"] = lens, _int(cu), _int(start, torch.int64)
    s["longest"], s["layer"] = max(lens) + 1, _layer(case, lens) if own else None
    at, seg, t, block = (_int(x, torch.int64) for x in _rows_of(lens, headroom))
    if case["kind"] == "q8_build":
        n, w = case["n"], _row_window(case)
        s["K"], s["V"] = randn(batch * (n + w), h, d).to(dt), randn(batch * (n + w), h, d).to(dt)
        # kept positions, ascending in every segment: evenly spread with a little noise, the window's rows last
        length = _int(lens, torch.int64)[seg]
        step = n / (length - w).clamp(min=1)
        pos = ((t + torch.rand(t.shape, generator=gen, device="cuda", dtype=torch.float64)) * step).long().clamp(max=n - 1)
        s["indices"] = torch.where(t >= length - w, n + w - (length - t), pos).to(torch.int32)
        s["at"], s["block"], s["head"] = at, block, seg % h
        s["from"] = s["indices"].long() + seg // h * (n + w)
    else:
        K, V = randn(len(at), d), randn(len(at), d)
    q8 = case["q8"] or case["kind"].startswith("q8")
    kept_as = F8 if q8 else dt
    s["K_cache"], s["V_cache"] = empty(rows, d, dtype=kept_as), empty(rows, d, dtype=kept_as)
    if q8:
        s["k_scale"], s["v_scale"] = (empty(blocks, dtype=torch.float32) for _ in range(2))
    s["seg_len"] = _int(lens)
    if case["kind"] == "q8_build":
        return s
    if q8:
        for name, x in (("K", K), ("V", V)):
            codes, scale = _quantise(x.to(dt).float(), block, blocks)
            s[name + "_cache"].view(torch.uint8)[at] = codes.view(torch.uint8)
            s[name.lower() + "_scale"].copy_(scale)
    else:
        s["K_cache"][at], s["V_cache"][at] = K.to(dt), V.to(dt)
    if case["kind"] == "move":
        s["picks"] = [int(v) for v in case["picks"].split()]
        lens_out = [lens[b * h + c] for b in s["picks"] for c in range(h)]
        _, _, rows_out, blocks_out = _layout(lens_out, case["new_headroom"])
        # (what a destination has where nothing is moved stays)
        s["K_out"], s["V_out"] = empty(rows_out, d, dtype=kept_as), empty(rows_out, d, dtype=kept_as)
        s["cu_out"], s["len_out"] = empty(len(lens_out) + 1, dtype=torch.int32), empty(len(lens_out), dtype=torch.int32)
        s["overflow"] = empty(1, dtype=torch.int32)
        s["segs"] = _int([b * h + c for b in s["picks"] for c in range(h)], torch.int64)
        if q8:
            s["k_scale_out"], s["v_scale_out"] = (empty(blocks_out, dtype=torch.float32) for _ in range(2))
        return s
    s["q"] = randn(batch, case["h_q"], d, by=2.0).to(dt)
    # a new row is larger than its block's others now and then
    big = torch.where(torch.rand((2, batch, h, 1), generator=gen, device="cuda") < 0.2, 4.0, 1.0)
    s["k"], s["v"] = (randn(batch, h, d) * big[0]).to(dt), (randn(batch, h, d) * big[1]).to(dt)
    s["turns"], s["turn"] = list(_int(lens).repeat(TURNS, 1).unbind(0)), 0
    s["overflow"] = empty(1, dtype=torch.int32)
    s["out"], s["lse"] = empty(batch, case["h_q"], d, dtype=torch.float32), empty(batch, case["h_q"], dtype=torch.float32)
    if own:
        import paper_2407_11550_amd as adakv
        s["ws"] = empty(adakv.decode_workspace_bytes(s["layer"], headroom), dtype=torch.uint8)
        s["cache"] = adakv.Q8Cache(s["K_cache"], s["V_cache"], s["k_scale"], s["v_scale"]) if q8 else None
    return s


# ---- the operators, plain ----------------------------------------------------------------------------------------
def _plain_prompt(s):
    case, g = s["case"], s["case"]["h_q"] // s["case"]["h_kv"]
    h, d, w, sinks = case["h_kv"], case["d"], s["row_lse"].shape[2], case["sinks"]
    first = 0
    for b, n in enumerate(s["lens"]):
        window = case["window"] or n
        K, V = (s[x][first:first + n].float().transpose(0, 1).contiguous() for x in "KV")          # [h, n, d]
        q = s["q"][first:first + n].float().view(n, h, g, d).permute(1, 2, 0, 3).contiguous()        # [h, g, n, d]
        lse = torch.empty((h, g, n), device="cuda")
        out = torch.empty((h, g, n, d), device="cuda")
        step = 1024
        for r0 in range(0, n, step):                 # (a piece of the rows at a time: the logits of all would not fit)
            r1 = min(n, r0 + step)
            lo = max(0, r0 - window + 1)
            j = torch.arange(lo, r1, device="cuda")
            if lo > 0 and sinks > 0:
                j = torch.cat([torch.arange(min(sinks, lo), device="cuda"), j])
            i = torch.arange(r0, r1, device="cuda")[:, None]
            seen = (j <= i) & ((j > i - window) | (j < sinks))
            x = torch.matmul(q[:, :, r0:r1].reshape(h, -1, d), K[:, j].transpose(1, 2)).view(h, g, r1 - r0, -1) / math.sqrt(d)
            x = x.masked_fill(~seen, -math.inf)
            top = x.amax(dim=-1, keepdim=True)
            x = torch.exp(x - top)
            total = x.sum(dim=-1, keepdim=True)
            out[:, :, r0:r1] = torch.matmul((x / total).view(h, -1, len(j)), V[:, j]).view(h, g, -1, d)
            lse[:, :, r0:r1] = (top + torch.log(total))[..., 0]
        s["out"][first:first + n] = out.permute(2, 0, 1, 3).reshape(n, h * g, d).to(s["out"].dtype)
        s["row_lse"][b] = lse.view(h * g, n)[:, n - w:]
        first += n
    return dict(out=s["out"], row_lse=s["row_lse"])


def _take(t, at):
    """Rows of a tensor; 8-bit ones by their codes."""
    return t.view(torch.uint8)[at].view(F8) if t.dtype == F8 else t[at]


def _put(t, at, x):
    if t.dtype == F8:
        t.view(torch.uint8)[at] = x.view(torch.uint8)
    else:
        t[at] = x


def _attend(q, K, V, seen, scale):
    """q [S, g, d] over rows [S, T, d] of which `seen` [S, T] count; 32 bits."""
    x = torch.matmul(q, K.transpose(1, 2)) * scale
    x = x.masked_fill(~seen[:, None], -math.inf)
    top = x.amax(dim=-1, keepdim=True)
    x = torch.exp(x - top)
    total = x.sum(dim=-1, keepdim=True)
    V = V.masked_fill(~seen[..., None], 0.0)
    return torch.matmul(x / total, V), (top + torch.log(total))[..., 0]


def _append_q8(codes, scale, start, held, room, new):
    """One row per segment into an 8-bit cache, in place: the open block takes the larger exponent."""
    where, blk = start + held, start // BLOCK + torch.arange(len(start), device="cuda") + held // BLOCK
    where, blk = where.clamp(max=len(codes) - 1), blk.clamp(max=len(scale) - 1)
    k_row, fresh = _exponent(_magnitude(new)), held % BLOCK == 0
    k_old = torch.where(fresh, k_row, _exponent_of(scale[blk]))
    k = torch.where(room, torch.maximum(k_old, k_row), k_old)
    t = torch.arange(BLOCK, device="cuda")
    rows = (start + held // BLOCK * BLOCK)[:, None] + t
    mine = (t < (held % BLOCK)[:, None]) & room[:, None]
    rows = torch.where(mine, rows, where[:, None])                # (nothing else of the block is touched)
    old = _take(codes, rows.reshape(-1)).view(len(start), BLOCK, -1).float()
    again = _round8(old * _pow2(k_old - k)[:, None, None])
    line = torch.where(room[:, None], _round8(new * _pow2(-k)[:, None]).float(), _take(codes, where).float()).to(F8)
    again = torch.where(mine[..., None], again.float(), line.float()[:, None]).to(F8)
    _put(codes, rows.reshape(-1), again.view(-1, again.shape[-1]))
    _put(codes, where, line)
    scale[blk] = torch.where(room, _pow2(k), scale[blk])


def _plain_step(s, lens):
    """window_step and q8_step: the new row joins its segment, then every query head looks at its segment's rows."""
    case = s["case"]
    h, d, S = case["h_kv"], case["d"], case["batch"] * case["h_kv"]
    g, q8 = case["h_q"] // h, case["kind"] == "q8_step"
    cap = s["cu"][1:].long() - s["cu"][:-1].long() + case["headroom"]
    held = lens.long()
    room = held < cap
    for name, new in (("K", s["k"]), ("V", s["v"])):
        cache, new = s[name + "_cache"], new.view(S, d)
        if q8:
            _append_q8(cache, s[name.lower() + "_scale"], s["start"], held, room, new.float())
        else:
            at = (s["start"] + held).clamp(max=len(cache) - 1)
            cache[at] = torch.where(room[:, None], new, cache[at])
    now = held + room
    s["overflow"] |= (~room).any()
    window, sinks = case["window"] or s["longest"], case["sinks"]
    if window + sinks < s["longest"]:                # the first rows and the last ones alone
        t = torch.arange(sinks + window, device="cuda").expand(S, -1)
        t = torch.where((t < sinks) | (now[:, None] <= sinks + window), t, t + now[:, None] - sinks - window)
    else:
        t = torch.arange(s["longest"], device="cuda").expand(S, -1)
    seen = t < now[:, None]
    at = (s["start"][:, None] + t).clamp(max=len(s["K_cache"]) - 1)
    K, V = (_take(s[x], at.reshape(-1)).view(S, -1, d).float() for x in ("K_cache", "V_cache"))
    if q8:
        blk = (s["start"] // BLOCK + torch.arange(S, device="cuda"))[:, None] + t // BLOCK
        blk = blk.clamp(max=len(s["k_scale"]) - 1)
        K, V = K * s["k_scale"][blk][..., None], V * s["v_scale"][blk][..., None]
    out, lse = _attend(s["q"].view(S, g, d).float(), K, V, seen, 1.0 / math.sqrt(d))
    lens.copy_(now)
    s["out"].copy_(out.view(s["out"].shape))
    s["lse"].copy_(lse.view(s["lse"].shape))


def _plain_build(s):
    for x in "KV":
        rows = s[x][s["from"], s["head"]].float()
        codes, scale = _quantise(rows, s["block"], len(s["k_scale"]))
        _put(s[x + "_cache"], s["at"], codes)
        s[x.lower() + "_scale"].copy_(scale)
    s["seg_len"].copy_(s["cu"][1:] - s["cu"][:-1])


def _plain_move(s):
    case, src = s["case"], s["segs"]
    sizes = (s["cu"][1:] - s["cu"][:-1]).long()[src]
    s["cu_out"][1:] = torch.cumsum(sizes, 0)
    new = case["new_headroom"]
    start = s["cu_out"][:-1].long() + new * torch.arange(len(src), device="cuda")
    lens = torch.minimum(s["seg_len"].long()[src], sizes + new)
    s["overflow"] |= (lens < s["seg_len"][src]).any()
    s["len_out"].copy_(lens)
    t = torch.arange(s["longest"], device="cuda")
    mine = t < lens[:, None]
    here, there = (start[:, None] + t)[mine], (s["start"][src][:, None] + t)[mine]
    for x in ("K", "V"):
        _put(s[x + "_out"], here, _take(s[x + "_cache"], there))
    if case["q8"]:
        t = torch.arange(s["longest"] // BLOCK + 1, device="cuda")
        mine = t * BLOCK < lens[:, None]
        order = torch.arange(len(src), device="cuda")
        here, there = ((start // BLOCK + order)[:, None] + t)[mine], ((s["start"][src] // BLOCK + src)[:, None] + t)[mine]
        for x in ("k_scale", "v_scale"):
            s[x + "_out"][here] = s[x][there]


def _own(s):
    import paper_2407_11550_amd as adakv
    case, layer = s["case"], s["layer"]
    kind, headroom = case["kind"], case.get("headroom")
    if kind == "prompt":
        window = case["window"] or max(s["lens"])
        adakv.window_attn(layer, s["q"], s["K"], s["V"], window, case["sinks"], out=s["out"], row_lse=s["row_lse"])
        return None
    if kind == "q8_build":
        cache = adakv.Q8Cache(s["K_cache"], s["V_cache"], s["k_scale"], s["v_scale"])
        adakv.cache_build_q8(layer, s["K"], s["V"], s["indices"], s["cu"], headroom, cache, s["seg_len"])
        return None
    if kind == "move":
        if case["q8"]:
            adakv.cache_move_q8(layer, s["picks"], s["cu"], headroom, adakv.Q8Cache(s["K_cache"], s["V_cache"], s["k_scale"], s["v_scale"]),
                                s["seg_len"], case["new_headroom"], s["cu_out"],
                                adakv.Q8Cache(s["K_out"], s["V_out"], s["k_scale_out"], s["v_scale_out"]), s["len_out"], s["overflow"])
        else:
            adakv.cache_move(layer, s["picks"], s["cu"], headroom, s["K_cache"], s["V_cache"], s["seg_len"], case["new_headroom"],
                             s["cu_out"], s["K_out"], s["V_out"], s["len_out"], s["overflow"])
        return None
    lens = s["turns"][s["turn"]]
    s["turn"] = (s["turn"] + 1) % TURNS
    if kind == "q8_step":
        adakv.decode_step_q8(layer, s["q"], s["k"], s["v"], s["cu"], headroom, s["cache"], lens, overflow=s["overflow"],
                             out=s["out"], lse=s["lse"], ws=s["ws"])
    else:
        adakv.decode_step(layer, s["q"], s["k"], s["v"], s["cu"], headroom, s["K_cache"], s["V_cache"], lens, overflow=s["overflow"],
                          out=s["out"], lse=s["lse"], ws=s["ws"], window=case["window"], sinks=case["sinks"])
    return lens


def run(s):
    kind, lens = s["case"]["kind"], None
    if own:
        lens = _own(s)
    elif kind == "prompt":
        _plain_prompt(s)
    elif kind == "q8_build":
        _plain_build(s)
    elif kind == "move":
        _plain_move(s)
    else:
        lens = s["turns"][s["turn"]]
        s["turn"] = (s["turn"] + 1) % TURNS
        _plain_step(s, lens)
    if kind == "prompt":
        return dict(out=s["out"], row_lse=s["row_lse"])
    names = ["K_cache", "V_cache"] + ["k_scale", "v_scale"] * (kind in ("q8_build", "q8_step"))
    if kind == "move":
        names = ["K_out", "V_out", "cu_out", "len_out", "overflow"] + ["k_scale_out", "v_scale_out"] * s["case"]["q8"]
    out = {x: s[x] for x in names}
    if kind == "q8_build":
        out["seg_len"] = s["seg_len"]
    if lens is not None:
        out.update(out=s["out"], lse=s["lse"], seg_len=lens, overflow=s["overflow"])
    return out


def _visible(n, window, sinks):
    """Pairs of a row and a key it sees, in a prompt of n tokens."""
    i = np.arange(n, dtype=np.int64)
    near = np.minimum(i + 1, window)
    return int((near + np.minimum(i + 1 - near, sinks)).sum())


def work(case):
    e = 4 if case["dtype"] == "fp32" else 2
    h_q, h, d, g = case["h_q"], case["h_kv"], case["d"], case["h_q"] // case["h_kv"]
    if case["kind"] == "prompt":
        lens = _prompt_lengths(case)
        pairs = sum(_visible(n, case["window"] or n, case["sinks"]) for n in lens)
        return dict(bytes=2 * sum(lens) * (h_q + h) * d * e + 4 * case["batch"] * h_q * _row_window(case), flops=4 * d * h_q * pairs)
    lens = _kept(case)
    S, rows = len(lens), sum(lens)
    blocks = sum((v + BLOCK - 1) // BLOCK for v in lens)
    if case["kind"] == "q8_build":
        return dict(bytes=rows * (2 * d * e + 2 * d + 4) + 8 * blocks + 8 * S, flops=0)
    if case["kind"] == "move":
        picks = [int(v) for v in case["picks"].split()]
        held = [sum(lens[b * h:(b + 1) * h]) for b in range(case["batch"])]
        row = 2 * d + 8 / BLOCK if case["q8"] else 2 * d * e
        return dict(bytes=row * (sum(held[b] for b in set(picks)) + sum(held[b] for b in picks)) + 8 * S + 8 * len(picks) * h, flops=0)
    io = case["batch"] * h_q * (d * e + 4 * d + 4) + S * 2 * d * e + 12 * S
    if case["kind"] == "q8_step":
        return dict(bytes=2 * d * (rows + 2 * S) + 8 * (blocks + S) + io, flops=4 * g * d * (rows + S))
    seen = sum(min(v + 1, case["window"] + case["sinks"]) for v in lens)
    return dict(bytes=2 * d * e * (seen + S) + io, flops=4 * g * d * seen)


# ---- the definitions, in 64 bits ---------------------------------------------------------------------------------
def _exact_rows(q, K, V, i, window, sinks):
    """Row by row softmax attention of q [r, d], the rows of positions i [r], over K, V [n, d]."""
    j = torch.arange(K.shape[0], device="cuda")
    dist = i[:, None] - j[None, :]
    hidden = (dist < 0) | ((dist >= window) & (j[None, :] >= sinks))
    logit = (q @ K.T.contiguous()) / math.sqrt(q.shape[1])
    logit[hidden] = -math.inf
    return torch.softmax(logit, dim=1) @ V, torch.logsumexp(logit, dim=1)


def _exact_prompt(s):
    case = s["case"]
    g, w = case["h_q"] // case["h_kv"], s["row_lse"].shape[2]
    out = torch.zeros(s["out"].shape, dtype=torch.float64, device="cuda")
    row_lse = torch.zeros(s["row_lse"].shape, dtype=torch.float64, device="cuda")
    first = 0
    for b, n in enumerate(s["lens"]):
        window = case["window"] or n
        for hq in range(case["h_q"]):
            q = s["q"][first:first + n, hq].double()
            K, V = s["K"][first:first + n, hq // g].double(), s["V"][first:first + n, hq // g].double()
            lse = torch.empty(n, dtype=torch.float64, device="cuda")
            for r in range(0, n, 4096):
                i = torch.arange(r, min(n, r + 4096), device="cuda")
                end = int(i[-1]) + 1
                # (keys behind the window of all these rows are left out where there are no sinks among them)
                cut = max(0, r - window + 1)
                keep = torch.cat([torch.arange(min(cut, case["sinks"]), device="cuda"), torch.arange(cut, end, device="cuda")])
                logit = (q[r:end] @ K[keep].T.contiguous()) / math.sqrt(case["d"])
                dist = i[:, None] - keep[None, :]
                logit[(dist < 0) | ((dist >= window) & (keep[None, :] >= case["sinks"]))] = -math.inf
                lse[r:end] = torch.logsumexp(logit, dim=1)
                out[first + r:first + end, hq] = torch.softmax(logit, dim=1) @ V[keep]
                del logit, dist
            row_lse[b, hq] = lse[n - w:]
        first += n
    return dict(out=out, row_lse=row_lse)


def _e4m3(x):
    """The nearest e4m3 value of numbers within its range, halves to the even one, in 64 bits."""
    mag = np.abs(x)
    _, e = np.frexp(mag)
    ulp = np.exp2(np.maximum(e - 4.0, -9.0))
    return np.copysign(np.round(mag / ulp) * ulp, x)


def _scale_exponent(m):
    if m == 0.0:
        return LOW_K
    k = math.ceil(math.log2(m / TOP))
    while TOP * 2.0 ** k < m:
        k += 1
    while TOP * 2.0 ** (k - 1) >= m:
        k -= 1
    return min(max(k, LOW_K), HIGH_K)


def _exact_build(s):
    headroom = s["case"]["headroom"]
    cu, start, rows, blocks = _layout(s["lens"], headroom)
    idx, h, out = s["indices"].cpu().numpy(), s["case"]["h_kv"], {}
    stride = s["case"]["n"] + _row_window(s["case"])
    for x in "KV":
        codes, scale = np.zeros((rows, s["case"]["d"])), np.zeros(blocks)
        data = s[x].float().cpu().numpy()
        for g, n in enumerate(s["lens"]):
            mine = data[idx[cu[g]:cu[g + 1]] + g // h * stride, g % h].astype(np.float64)
            for t in range(0, n, BLOCK):
                piece = mine[t:t + BLOCK]
                k = _scale_exponent(float(np.abs(piece).max()))
                codes[start[g] + t:start[g] + t + len(piece)] = _e4m3(piece / 2.0 ** k)
                scale[start[g] // BLOCK + g + t // BLOCK] = 2.0 ** k
        out[x + "_cache"], out[x.lower() + "_scale"] = torch.from_numpy(codes), torch.from_numpy(scale)
    return dict(out, seg_len=None)


def _exact_step(s):
    case, headroom = s["case"], s["case"]["headroom"]
    h, d, q8 = case["h_kv"], case["d"], case["kind"] == "q8_step"
    g = case["h_q"] // h
    _, start, _, _ = _layout(s["lens"], headroom)
    state = {}
    for x in "KV":
        state[x] = s[x + "_cache"].double()
        if q8:
            state[x + "s"] = s[x.lower() + "_scale"].double()
    out = torch.zeros(s["out"].shape, dtype=torch.float64, device="cuda")
    lse = torch.zeros(s["lse"].shape, dtype=torch.float64, device="cuda")
    for seg, n in enumerate(s["lens"]):
        b, c, a = seg // h, seg % h, int(start[seg])
        rows = {}
        for x, new in (("K", s["k"]), ("V", s["v"])):
            new = new[b, c].double()
            if not q8:
                state[x][a + n] = new
                rows[x] = state[x][a:a + n + 1]
                continue
            at = a // BLOCK + seg + n // BLOCK
            k_row, t0 = _scale_exponent(float(new.abs().max())), n // BLOCK * BLOCK
            k = k_row if n % BLOCK == 0 else max(k_row, int(round(math.log2(float(state[x + "s"][at])))))
            if n % BLOCK:
                old = state[x][a + t0:a + n].cpu().numpy() * float(state[x + "s"][at])
                state[x][a + t0:a + n] = torch.from_numpy(_e4m3(old / 2.0 ** k)).cuda()
            state[x][a + n] = torch.from_numpy(_e4m3(new.cpu().numpy() / 2.0 ** k)).cuda()
            state[x + "s"][at] = 2.0 ** k
            blocks = state[x + "s"][a // BLOCK + seg:a // BLOCK + seg + n // BLOCK + 1]
            rows[x] = state[x][a:a + n + 1] * blocks.repeat_interleave(BLOCK)[:n + 1, None]
        i = torch.full((g,), n, device="cuda")
        o, z = _exact_rows(s["q"][b, c * g:(c + 1) * g].double(), rows["K"], rows["V"], i, case["window"] or n + 1, case["sinks"])
        out[b, c * g:(c + 1) * g], lse[b, c * g:(c + 1) * g] = o, z
    done = dict(out=out, lse=lse, K_cache=None, V_cache=None, seg_len=None, overflow=None)
    if q8:
        done.update(K_cache=state["K"], V_cache=state["V"], k_scale=state["Ks"], v_scale=state["Vs"])
    return done


def exact(case, seed):
    if case["kind"] == "move":
        return None                                  # copied rows and whole numbers
    global own
    was, own = own, False
    try:
        s = prepare(case, seed)
    finally:
        own = was
    return {"prompt": _exact_prompt, "q8_build": _exact_build}.get(case["kind"], _exact_step)(s)

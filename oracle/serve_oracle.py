"""Plain fp64 CPU oracle for what surrounds a compressed cache: attention limited to a window and sinks, the cache
in 8 bits, sequences of a cache moved.

THIS IS TEST INFRASTRUCTURE, NOT THE PRODUCT.  It shares no code with the HIP path and never imports the
package that wraps the HIP library.  Notation as in decode_oracle.py.

Readings:
    W1  a row sees the keys at most window - 1 places before it, and the first `sinks` keys however far back;
        never a later key.  A hidden key has no part in the row's result, whatever its key and value are.
    W2  in a decoding step the row is the segment's last one: with len rows held it sees t < sinks and
        t >= len - window.
    Q1  a block is 32 rows of a segment counted from its first; its scale is the smallest power of two 2^k with every
        finite magnitude <= 448 * 2^k, -60 <= k <= 100.
    Q2  values are rounded to nearest e4m3, halves to even; beyond 448 * 2^100 they saturate; what is not finite is NaN.
    Q3  a row appended to a block with rows in it takes the larger of the block's k and its own; if that is its own, the
        block's rows are rounded again to it.
    M1  capacities, lengths and rows move with a sequence; rows beyond a smaller capacity are left out and reported.
"""
from __future__ import annotations

import math

import numpy as np

from . import decode_oracle as D

BLOCK, TOP, LOW, HIGH = 32, 448.0, -60, 100


# ---- attention with a window ------------------------------------------------------------------------------
def visible(i, n, window, sinks):
    """The keys that row i of a sequence sees, among the first n."""
    j = np.arange(n)
    return (j <= i) & ((j > i - window) | (j < sinks))


def attend(q, K, V, scale):
    """One query row over the rows it sees: (output, log-sum-exp, weighted magnitudes of V, largest sum of |q k|)."""
    q, K, V = (np.asarray(x, dtype=np.float64) for x in (q, K, V))
    logit = scale * (K @ q)
    top = logit.max()
    e = np.exp(logit - top)
    a = e / e.sum()
    return a @ V, top + math.log(e.sum()), a @ np.abs(V), scale * (np.abs(K) @ np.abs(q)).max()


def prompt(q, K, V, window, sinks, scale):
    """Causal attention of one head: q, K, V [n, d].  Rows of what `attend` gives, stacked."""
    rows = []
    for i in range(len(q)):
        see = visible(i, len(K), window, sinks)
        rows.append(attend(q[i], K[see], V[see], scale))
    out, lse, mag, big = zip(*rows)
    return np.stack(out), np.array(lse), np.stack(mag), np.array(big)


def step_rows(length, window, sinks):
    """Rows of a segment of `length` rows that a decoding step looks at."""
    t = np.arange(length)
    return t[(t < sinks) | (t >= length - window)]


# ---- 8 bits ---------------------------------------------------------------------------------------------
def exponent(m):
    """Q1 for a largest finite magnitude m."""
    if m == 0.0:
        return LOW
    k = LOW
    while k < HIGH and TOP * 2.0 ** k < m:
        k += 1
    return k


def round_e4m3(x):
    """The nearest e4m3 number (4 significant bits, multiples of 2^-9 at least), halves to even; Q2 beyond the range."""
    x = np.asarray(x, dtype=np.float64)
    with np.errstate(invalid="ignore"):
        mag = np.minimum(np.abs(x), TOP)
        unit = np.exp2(np.maximum(np.floor(np.log2(np.where(mag > 0, mag, 1.0))) - 3, -9))
        y = np.minimum(np.round(mag / unit) * unit, TOP)
        return np.where(np.isfinite(x), np.copysign(y, x), np.nan)


def quantise(rows):
    """Rows of one segment -> (codes as numbers, exponents of its blocks)."""
    rows = np.asarray(rows, dtype=np.float64)
    codes, ks = np.empty(rows.shape), []
    for t in range(0, len(rows), BLOCK):
        piece = rows[t:t + BLOCK]
        ks.append(exponent(np.max(np.abs(piece), where=np.isfinite(piece), initial=0.0)))
        codes[t:t + BLOCK] = round_e4m3(piece * 2.0 ** -ks[-1])
    return codes, ks


def append(codes, ks, row):
    """Q3: one row behind a segment's codes; returns the new (codes, exponents)."""
    row = np.asarray(row, dtype=np.float64)
    own = exponent(np.max(np.abs(row), where=np.isfinite(row), initial=0.0))
    t0, ks = len(codes) // BLOCK * BLOCK, list(ks)
    if len(codes) == t0:
        ks.append(own)
    elif own > ks[-1]:
        codes = np.concatenate([codes[:t0], round_e4m3(codes[t0:] * 2.0 ** (ks[-1] - own))])
        ks[-1] = own
    return np.concatenate([codes, round_e4m3(row * 2.0 ** -ks[-1])[None]]), ks


def values(codes, ks):
    """What a segment's codes stand for."""
    return codes * np.repeat(np.exp2(np.array(ks, dtype=np.float64)), BLOCK)[:len(codes), None]


def scale_places(cu_seqlens, headroom):
    """Where each segment's first scale is."""
    start = D.segment_starts(cu_seqlens, headroom)
    return start // BLOCK + np.arange(len(start))


# ---- moving ---------------------------------------------------------------------------------------------
def move(picks, h, cu_seqlens, headroom, lens, headroom_out):
    """M1: (cu_out, lens_out, [(source row, destination row, rows)] per destination segment, overflow)."""
    cu, start = np.asarray(cu_seqlens, dtype=np.int64), D.segment_starts(cu_seqlens, headroom)
    src = [b * h + c for b in picks for c in range(h)]
    cu_out = np.concatenate([[0], np.cumsum([cu[s + 1] - cu[s] for s in src])])
    start_out, cap = D.segment_starts(cu_out, headroom_out), D.segment_caps(cu_out, headroom_out)
    lens_out = np.minimum([lens[s] for s in src], cap)
    return (cu_out, lens_out, [(int(start[s]), int(start_out[i]), int(lens_out[i])) for i, s in enumerate(src)],
            bool(np.any(lens_out < [lens[s] for s in src])))

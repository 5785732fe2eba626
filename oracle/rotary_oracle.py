"""Plain fp64 CPU oracle for what stands in front of attention: heads turned by their positions, and their norms.

THIS IS TEST INFRASTRUCTURE, NOT THE PRODUCT.  It shares no code with the HIP path and never imports the package
that wraps the HIP library.

Readings:
    R1  pair i < dims/2 of a head are its elements i and i + dims/2 (half) or 2i and 2i + 1 (interleaved); elements from
        dims on stay.
    R2  frequency i is base^(-2i/dims); scaled for contexts `factor` times as long: all divided by it (linear); the base
        times factor^(dims/(dims-2)) (base); or (parts) with r = original_len * f / 2 pi turns within the original
        length, kept from `high` turns on, divided by the factor up to `low` turns, and mixed linearly in r between.
    R3  a norm divides a head by the root of the mean of its squares plus eps and multiplies it by a weight per element,
        before it is turned.
"""
from __future__ import annotations

import numpy as np


def frequencies(dims, base=10000.0, scaling="none", factor=1.0, original_len=0, low=1.0, high=4.0):
    i = np.arange(dims // 2, dtype=np.float64)
    if scaling == "base" and dims > 2:
        base = base * factor ** (dims / (dims - 2))
    f = np.exp(-2.0 * i / dims * np.log(base))
    if scaling == "linear":
        return f / factor
    if scaling == "parts":
        u = np.clip((original_len * f / (2 * np.pi) - low) / (high - low), 0.0, 1.0)
        return u * f + (1 - u) * f / factor
    return f


def turn(x, positions, freq, dims, layout, magnitude=1.0):
    """x [rows, heads, d] at positions [rows]."""
    x = np.asarray(x, dtype=np.float64)
    t = np.asarray(positions, dtype=np.float64)[:, None, None] * np.asarray(freq, dtype=np.float64)
    cos, sin = np.cos(t), np.sin(t)
    first = np.arange(dims // 2) if layout == "half" else 2 * np.arange(dims // 2)
    second = first + (dims // 2 if layout == "half" else 1)
    y = x.copy()
    y[..., first] = magnitude * (x[..., first] * cos - x[..., second] * sin)
    y[..., second] = magnitude * (x[..., second] * cos + x[..., first] * sin)
    return y


def norm(x, weight, eps):
    x = np.asarray(x, dtype=np.float64)
    return x / np.sqrt((x ** 2).mean(-1, keepdims=True) + eps) * np.asarray(weight, dtype=np.float64)

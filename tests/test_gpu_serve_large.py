"""Caches whose rows lie beyond 32-bit offsets, and prompts with rows as far apart as the call takes them."""
import math

import numpy as np
import pytest
import torch

import paper_2407_11550_amd as adakv
from oracle import decode_oracle as D
from oracle import serve_oracle as S
from serve_util import DEV, assert_within, attention_bound, f64, lse_bound, offsets

pytestmark = pytest.mark.gpu
BF = torch.bfloat16
G, H, DIM, LENS = 4, 3, 128, [40, 75, 300]


def layer_of(lens):
    return adakv.Layer(BF, G * H, H, DIM, 1, 7, 0.2, [max(lens)], [sum(lens)])


def randn(seed, *shape):
    return torch.randn(shape, generator=torch.Generator().manual_seed(seed)).to(BF).to(DEV)


def check(q, rows_k, rows_v, out, lse):
    for s in range(H):
        K, V = rows_k[s], rows_v[s]
        for i in range(G):
            ref, z, mag, big = S.attend(f64(q[0, s * G + i]), K, V, 1 / math.sqrt(DIM))
            keys = np.array(len(K))
            assert_within(f64(out[0, s * G + i]), ref, attention_bound(BF, DIM, ref, mag, np.array(big), np.array(z), keys, rounded=False), f"segment {s}")
            assert_within(f64(lse[0, s * G + i]), z, lse_bound(DIM, np.array(big), np.array(z), keys), f"lse {s}")


def test_a_windowed_step_beyond_four_gigabytes():
    """The last segment starts 6.1 GB into each tensor."""
    hr, window, sinks = 12_000_000, 90, 7
    layer, cu = layer_of(LENS), offsets(LENS)
    start = D.segment_starts(cu, hr)
    assert start[-1] * DIM * 2 > 2 ** 32
    K, V = (torch.empty((adakv.cache_rows(layer, hr), DIM), dtype=BF, device=DEV) for _ in range(2))
    for s, a in enumerate(start):
        K[a:a + LENS[s]], V[a:a + LENS[s]] = randn(s, LENS[s], DIM), randn(10 + s, LENS[s], DIM)
    q, kn, vn = randn(20, 1, G * H, DIM), randn(21, 1, H, DIM), randn(22, 1, H, DIM)
    cu_t, lens = (torch.tensor(x, dtype=torch.int32, device=DEV) for x in (cu, LENS))
    out, lse = adakv.decode_step(layer, q, kn, vn, cu_t, hr, K, V, lens, want_lse=True, window=window, sinks=sinks)
    torch.cuda.synchronize()
    assert lens.tolist() == [n + 1 for n in LENS]
    seen = [a + S.step_rows(n + 1, window, sinks) for a, n in zip(start, LENS)]
    check(q, *([f64(t[torch.as_tensor(rows, device=DEV)]) for rows in seen] for t in (K, V)), out, lse)


def test_an_8_bit_cache_beyond_four_gigabytes_built_stepped_and_moved():
    hr = 18_000_000
    layer, cu = layer_of(LENS), offsets(LENS)
    start, place = D.segment_starts(cu, hr), S.scale_places(cu, hr)
    assert start[-1] * DIM > 2 ** 32
    K, V = randn(1, 301, H, DIM), randn(2, 301, H, DIM)
    cu_t = torch.tensor(cu, dtype=torch.int32, device=DEV)
    idx = torch.cat([torch.arange(n, dtype=torch.int32) for n in LENS]).to(DEV)
    rows, scales = adakv.cache_rows(layer, hr), adakv.q8_scales(layer, hr)
    cache = adakv.Q8Cache(*(torch.empty((rows, DIM), dtype=torch.uint8, device=DEV).view(torch.float8_e4m3fn) for _ in range(2)),
                          *(torch.empty(scales, dtype=torch.float32, device=DEV) for _ in range(2)))
    cache, lens = adakv.cache_build_q8(layer, K, V, idx, cu_t, hr, cache)
    q, kn, vn = randn(20, 1, G * H, DIM), randn(21, 1, H, DIM) * 4, randn(22, 1, H, DIM)
    out, lse = adakv.decode_step_q8(layer, q, kn, vn, cu_t, hr, cache, lens, want_lse=True)
    torch.cuda.synchronize()
    want = {}
    for name, x, new in (("K", K, kn), ("V", V, vn)):
        want[name] = [S.append(*S.quantise(f64(x[:LENS[s], s])), f64(new[0, s])) for s in range(H)]
        codes, scale = (cache.K, cache.k_scale) if name == "K" else (cache.V, cache.v_scale)
        for s in range(H):
            c, ks = want[name][s]
            got = codes.view(torch.uint8)[start[s]:start[s] + len(c)].view(torch.float8_e4m3fn)
            assert np.array_equal(f64(got.float()), c), (name, s)
            assert np.array_equal(f64(scale[place[s]:place[s] + len(ks)]), np.exp2(np.array(ks, dtype=float)))
    check(q, [S.values(*x) for x in want["K"]], [S.values(*x) for x in want["V"]], out, lse)
    # out of the far segments and into them
    to, cu2, near, len2 = adakv.cache_move_q8(layer, [0], cu_t, hr, cache, lens, 5)
    far = adakv.Q8Cache(*(torch.zeros_like(t.view(torch.uint8)).view(t.dtype) for t in cache))
    _, cu3, far, len3 = adakv.cache_move_q8(to, [0], cu2, 5, near, len2, hr, out=far)
    torch.cuda.synchronize()
    assert torch.equal(cu3, cu_t) and torch.equal(len3, lens)
    for s in range(H):
        for a, b in zip(cache[:2], far[:2]):
            at = slice(start[s], start[s] + LENS[s] + 1)
            assert torch.equal(a.view(torch.uint8)[at], b.view(torch.uint8)[at])
        at = slice(place[s], place[s] + -(-(LENS[s] + 1) // 32))
        for a, b in zip(cache[2:], far[2:]):
            assert torch.equal(a[at], b[at])


@pytest.mark.parametrize("dtype,h_q", [(BF, 2), (BF, 66), (torch.float32, 2)])
def test_prompt_rows_far_apart(dtype, h_q):
    """Keys just under 16 MiB apart: a sequence of 300 rows spans 5 GB."""
    n, d, w = 300, 64, 4
    step = (1 << 24) // torch.empty((), dtype=dtype).element_size() - 64
    K, V = (torch.empty((n - 1) * step + d, dtype=dtype, device=DEV).as_strided((n, 1, d), (step, d, 1)) for _ in range(2))
    x = [torch.randn((n, k, d), generator=torch.Generator().manual_seed(k)).to(dtype).to(DEV) for k in (h_q, 1, 1)]
    K.copy_(x[1])
    V.copy_(x[2])
    layer = adakv.Layer(dtype, h_q, 1, d, w, 7, 0.2, [n - w], [w], k_strides=(step, d), v_strides=(step, d))
    near = adakv.Layer(dtype, h_q, 1, d, w, 7, 0.2, [n - w], [w])
    for window in (n, 33):
        a = adakv.window_attn(layer, x[0], K, V, window, 2)
        b = adakv.window_attn(near, x[0], x[1], x[2], window, 2)
        torch.cuda.synchronize()
        assert torch.equal(a, b)

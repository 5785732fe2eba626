"""Attention where the numbers end: logits that are no numbers or infinite, rows that no weight is left for, values near the
end of their type."""
import math

import numpy as np
import pytest
import torch

import paper_2407_11550_amd as adakv
from oracle import serve_oracle as S
from serve_util import DEV, assert_within, attention_bound, f64, lse_bound
from test_gpu_decode_window import cache
from test_gpu_q8 import build

pytestmark = pytest.mark.gpu
BF, FH, FS = torch.bfloat16, torch.float16, torch.float32

# (lengths, window): a segment by one workgroup, in parts; the same two without a window
DIVISIONS = {"one_workgroup": ([900, 61], 100), "parts": ([2500, 61], 1500), "short": ([150, 61], None), "long": ([2500, 61], None)}


@pytest.mark.parametrize("div", DIVISIONS, ids=str)
@pytest.mark.parametrize("dtype, g, d", [(BF, 4, 128), (BF, 1, 64), (FH, 8, 64), (FS, 4, 128)])
@pytest.mark.parametrize("sign", [1.0, -1.0])
def test_a_step_over_infinite_keys(div, dtype, g, d, sign):
    """A logit of -inf has weight 0; where the visible rows have no other the result is none: NaN, and ln 0."""
    lens, window = DIVISIONS[div]
    kw = {} if window is None else dict(window=window, sinks=2)
    layer, K, V, cu, seg_len, q, _, _ = cache(dtype, g, 2, d, lens, 3)
    q = sign * (q.abs() + 1.0)
    K[lens[0] - 7] = -sign * float("inf")
    out, lse = adakv.decode_attn(layer, q, cu, 3, K, V, seg_len, want_lse=True, **kw)
    torch.cuda.synchronize()
    see = S.step_rows(lens[0], window or lens[0], 2)
    see = see[see != lens[0] - 7]
    for i in range(g):
        ref, z, mag, big = S.attend(f64(q[0, i]), f64(K[see]), f64(V[see]), 1 / math.sqrt(d))
        keys = np.array(len(see))
        assert_within(f64(out[0, i]), ref, attention_bound(dtype, d, ref, mag, np.array(big), np.array(z), keys, rounded=False), f"head {i}")
        assert_within(f64(lse[0, i]), z, lse_bound(d, np.array(big), np.array(z), keys), f"lse {i}")
    K[:lens[0]] = -sign * float("inf")
    out, lse = adakv.decode_attn(layer, q, cu, 3, K, V, seg_len, want_lse=True, **kw)
    torch.cuda.synchronize()
    assert torch.isnan(out[0, :g]).all() and torch.isneginf(lse[0, :g]).all()
    assert torch.isfinite(out[0, g:]).all() and torch.isfinite(lse[0, g:]).all()


@pytest.mark.parametrize("lens", [[150, 61], [2500, 61]], ids=["one_workgroup", "parts"])
@pytest.mark.parametrize("dtype, g, d", [(BF, 4, 128), (BF, 1, 64), (FH, 8, 64), (FS, 4, 128)])
@pytest.mark.parametrize("what", [float("nan"), float("inf")])
def test_a_key_that_is_no_number_is_not_passed_over_without_a_window(dtype, g, d, lens, what):
    layer, K, V, cu, seg_len, q, _, _ = cache(dtype, g, 2, d, lens, 3)
    K[lens[0] - 1] = what
    out, lse = adakv.decode_attn(layer, q.abs() + 1.0, cu, 3, K, V, seg_len, want_lse=True)
    torch.cuda.synchronize()
    assert torch.isnan(out[0, :g]).all() and torch.isnan(lse[0, :g]).all()
    assert torch.isfinite(out[0, g:]).all() and torch.isfinite(lse[0, g:]).all()


@pytest.mark.parametrize("lens", [[250, 61], [1700, 40]], ids=["one_workgroup", "parts"])
@pytest.mark.parametrize("dtype, g, d", [(BF, 4, 128), (FH, 8, 64)])
def test_an_8_bit_step_whose_logits_are_all_minus_infinity(dtype, g, d, lens):
    layer, cache8, cu, seg_len, _ = build(dtype, g, 2, d, lens, 4)
    codes = cache8.K.view(torch.uint8)
    codes[:lens[0], 5] = 0x38                     # 1
    q = torch.zeros((1, 2 * g, d), dtype=dtype, device=DEV)
    q[:, :, 5] = 1.0
    q[:, :g, 5] = -float("inf")
    q[:, :g, [c for c in range(d) if c != 5]] = 1.0
    codes[:lens[0]][codes[:lens[0]] == 0x7f] = 0
    out, lse = adakv.decode_attn_q8(layer, q, cu, 4, cache8, seg_len, want_lse=True)
    torch.cuda.synchronize()
    assert torch.isnan(out[0, :g]).all() and torch.isneginf(lse[0, :g]).all()
    assert torch.isfinite(out[0, g:]).all() and torch.isfinite(lse[0, g:]).all()


@pytest.mark.parametrize("dtype", [BF, FH, FS])
@pytest.mark.parametrize("n", [7, 40])
def test_an_8_bit_step_with_a_scale_next_to_zero(dtype, n):
    """scale * 2^k of a block of zeros is below the fp32 range: all weights are alike, and rows past the end have none."""
    layer = adakv.Layer(dtype, 2, 1, 64, 1, 7, 0.2, [n], [n], scale=1e-30)
    cache8 = adakv.q8_cache(layer, 3, DEV)
    cu, seg_len = torch.tensor([0, n], dtype=torch.int32, device=DEV), torch.tensor([n], dtype=torch.int32, device=DEV)
    for s in cache8[2:]:
        s.fill_(2.0 ** -60)
    cache8.v_scale.fill_(1.0)
    cache8.V.view(torch.uint8)[:n] = 0x38         # ones
    q = torch.ones((1, 2, 64), dtype=dtype, device=DEV)
    out, lse = adakv.decode_attn_q8(layer, q, cu, 3, cache8, seg_len, want_lse=True)
    torch.cuda.synchronize()
    assert (out == 1.0).all()
    # (ln n by log2 and a multiplication: two roundings of log2, one of the constant and one of the product)
    assert np.abs(f64(lse) - math.log(n)).max() <= 5 * 2.0 ** -24 * math.log(n)


@pytest.mark.parametrize("cu", [[1 << 20, 40, 70], [40, 10, 70], [0, 1 << 20, 70], [-(1 << 31), 40, 70], [33, 40, 1 << 20], [0, -70, 70], [70, 70, 0]], ids=str)
def test_an_8_bit_build_stays_inside_with_corrupt_offsets(cu):
    """Offsets that are no running sum: nothing around the cache, its scales and the lengths is written."""
    print(cu, flush=True)
    h, hr, w, d, rows = 2, 5, 2, 64, 70
    layer = adakv.Layer(BF, h, h, d, w, 7, 0.2, [98], [rows])
    K = torch.randn((100, h, d), device=DEV).to(BF)
    idx = torch.arange(rows, dtype=torch.int32, device=DEV)
    held, scales, pad = adakv.cache_rows(layer, hr), adakv.q8_scales(layer, hr), 4096
    big = [torch.full((held + 2 * pad, d), 0x55, dtype=torch.uint8, device=DEV) for _ in range(2)]
    big += [torch.full((scales + 2 * pad,), 7.0, device=DEV) for _ in range(2)]
    lens = torch.full((h + 2 * pad,), 7, dtype=torch.int32, device=DEV)
    inside = [t[pad:len(t) - pad] for t in big]
    cache8 = adakv.Q8Cache(*(t.view(torch.float8_e4m3fn) for t in inside[:2]), *inside[2:])
    adakv.cache_build_q8(layer, K, K, idx, torch.tensor(cu, dtype=torch.int32, device=DEV), hr, cache8, lens[pad:pad + h])
    torch.cuda.synchronize()
    for t, fill in zip((*big, lens), (0x55, 0x55, 7, 7, 7)):
        assert (t[:pad] == fill).all() and (t[-pad:] == fill).all()


# ---- prompts -----------------------------------------------------------------------------------------------
def prompt(dtype, h_q, h, d, lens, seed=0):
    w = 2
    layer = adakv.Layer(dtype, h_q, h, d, w, 7, 0.2, [n - w for n in lens], [w * h for _ in lens])
    g = torch.Generator().manual_seed(seed)
    return layer, *((torch.randn((sum(lens), k, d), generator=g) * f).to(dtype).to(DEV) for k, f in ((h_q, 2.0), (h, 1.0), (h, 1.0)))


# query heads that make rows shared by four wavefronts, by two and by none
SHARES = [(2, 260), (3, 260), (70, 260), (70, 500), (70, 1100)]


@pytest.mark.parametrize("dtype, d", [(BF, 64), (BF, 128), (FH, 64), (FH, 128), (FS, 64), (FS, 128)])
@pytest.mark.parametrize("h_q, n", SHARES[:4])
def test_a_prompt_row_that_sees_infinite_keys_alone(dtype, d, h_q, n):
    """Logits of -inf: weight 0 beside others, NaN and ln 0 where there are no others."""
    layer, q, K, V = prompt(dtype, h_q, 1, d, [n])
    q, at = q.abs() + 1.0, n - 1
    window = 3
    K[at - 1:] = -float("inf")                    # the last row sees n - 3 and these two, the one before n - 4, n - 3 and one
    out, lse = adakv.window_attn(layer, q, K, V, window, want_lse=True)
    torch.cuda.synchronize()
    for hq in (0, h_q - 1):
        for k, i in enumerate((n - 2, n - 1)):
            see = np.arange(i - 2, n - 2)
            ref, z, mag, big = S.attend(f64(q[i, hq]), f64(K[see, 0]), f64(V[see, 0]), 1 / math.sqrt(d))
            keys = np.array(len(see))
            assert_within(f64(out[i, hq]), ref, attention_bound(dtype, d, ref, mag, np.array(big), np.array(z), keys, rounded=True), f"row {i}")
            assert_within(f64(lse[0, hq, k]), z, lse_bound(d, np.array(big), np.array(z), keys), f"lse {i}")
    out, lse = adakv.window_attn(layer, q, K, V, 2, want_lse=True)
    torch.cuda.synchronize()
    assert torch.isnan(out[n - 1].float()).all() and torch.isneginf(lse[0, :, 1]).all()
    assert torch.isfinite(out[:n - 1].float()).all() and torch.isfinite(lse[0, :, 0]).all()


@pytest.mark.parametrize("dtype, d", [(BF, 64), (BF, 128), (FS, 64), (FS, 128)])
@pytest.mark.parametrize("h_q, n", SHARES)
@pytest.mark.parametrize("hidden", [False, True])
def test_prompt_values_near_the_end_of_their_type(dtype, d, h_q, n, hidden):
    """Values from half the type's largest to all of it, of one sign or of both: a weighted mean of them is a number of the type.
    `hidden`: beside a value that is none and that few rows see."""
    layer, q, K, V = prompt(dtype, h_q, 1, d, [n])
    top = torch.finfo(dtype).max
    V = ((0.5 + 0.45 * torch.rand(V.shape, generator=torch.Generator().manual_seed(2))).to(DEV) * top).to(dtype)
    V[:, :, 1::2] *= torch.where(torch.arange(n, device=DEV) % 3 == 0, -1.0, 1.0).to(dtype)[:, None, None]
    window, sinks, at = (90, 3, 64) if hidden else (n, 0, n)
    clean = V.clone()
    if hidden:
        V[at] = float("nan")
    out, lse = adakv.window_attn(layer, q, K, V, window, sinks, want_lse=True)
    torch.cuda.synchronize()
    rows = np.array([i for i in range(n) if not at <= i < at + window])
    assert torch.isnan(out[at:at + window].float()).all()
    keys = np.array([S.visible(i, n, window, sinks).sum() for i in range(n)])
    for hq in sorted({0, h_q - 1}):
        ref, z, mag, big = S.prompt(f64(q[:, hq]), f64(K[:, 0]), f64(clean[:, 0]), window, sinks, 1 / math.sqrt(d))
        bound = attention_bound(dtype, d, ref, mag, big, z, keys, rounded=True)
        assert_within(f64(out[:, hq])[rows], ref[rows], bound[rows], f"head {hq}")
        assert_within(f64(lse[0, hq]), z[n - 2:], lse_bound(d, big, z, keys)[n - 2:], f"lse {hq}")

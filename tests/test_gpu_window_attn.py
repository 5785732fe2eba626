"""Attention over prompts with a window and sinks against 64 bits, and what it must leave alone."""
import math

import numpy as np
import pytest
import torch

import paper_2407_11550_amd as adakv
from oracle import serve_oracle as S
from serve_util import DEV, assert_within, attention_bound, f64, lse_bound

pytestmark = pytest.mark.gpu
BF, FH, FS = torch.bfloat16, torch.float16, torch.float32


def layer_of(dtype, h_q, h, d, lens, w, **kw):
    return adakv.Layer(dtype, h_q, h, d, w, 7, 0.2, [n - w for n in lens], [w * h for _ in lens], **kw)


def inputs(dtype, h_q, h, d, tokens, seed=0, by=2.0):
    g = torch.Generator().manual_seed(seed)
    return tuple((torch.randn((tokens, k, d), generator=g) * f).to(dtype).to(DEV) for k, f in ((h_q, by), (h, 1.0), (h, 1.0)))


def check(layer, q, K, V, window, sinks, out, row_lse, heads=None, what=""):
    """Every row of the named query heads (all of them by default) against 64 bits."""
    d, g, w = layer.d, layer.h_q // layer.h_kv, layer.w
    scale = layer.scale or 1.0 / math.sqrt(d)
    for b in range(layer.batch):
        n, t0 = layer.n[b] + w, layer.tok_off[b]
        keys = np.array([S.visible(i, n, window, sinks).sum() for i in range(n)])
        for hq in heads or range(layer.h_q):
            c = hq // g
            ref, lse, mag, big = S.prompt(f64(q[t0:t0 + n, hq]), f64(K[t0:t0 + n, c]), f64(V[t0:t0 + n, c]), window, sinks, scale)
            bound = attention_bound(layer.torch_dtype, d, ref, mag, big, lse, keys, rounded=True)
            assert_within(f64(out[t0:t0 + n, hq]), ref, bound, f"{what} sequence {b} head {hq}")
            if row_lse is not None:
                assert_within(f64(row_lse[b, hq]), lse[n - w:], lse_bound(d, big, lse, keys)[n - w:], f"{what} lse {b} {hq}")


CASES = [
    # dtype h_q h_kv d  lengths            w  window sinks
    (BF, 2, 1, 128, [2], 1, 1, 0),
    (BF, 4, 2, 128, [33, 2, 64], 1, 5, 1),
    (BF, 2, 2, 64, [127, 128, 129], 8, 64, 4),
    (BF, 8, 1, 128, [257], 32, 2 ** 31 - 1, 0),
    (BF, 4, 4, 128, [300, 65], 32, 63, 70),
    (BF, 3, 1, 64, [400], 3, 100, 400),          # sinks cover everything
    (FH, 2, 1, 128, [130, 31], 5, 32, 3),
    (FH, 4, 2, 64, [385], 32, 129, 64),
    (FH, 2, 2, 128, [258], 32, 258, 0),
    (FS, 2, 1, 64, [97, 3], 2, 31, 2),
    (FS, 2, 2, 128, [200, 129], 32, 2 ** 31 - 1, 2 ** 31 - 1),
    (FS, 4, 1, 128, [161], 16, 1, 33),
    (BF, 5, 5, 128, [200], 7, 1, 0),             # a row sees itself alone
    (BF, 2, 1, 128, [1500], 32, 65, 5),          # far rows: tiles between sinks and window are not visited
    # rows shared by one, two and four wavefronts, in every type and width (which of them goes by the number of workgroups)
    (BF, 64, 64, 128, [330, 33], 32, 200, 3),    # 256 workgroups of 128 rows
    (FH, 64, 64, 64, [330, 33], 32, 200, 3),
    (BF, 64, 64, 64, [300, 160], 7, 129, 0),     # 320
    (FH, 64, 64, 128, [300, 160], 7, 129, 0),
    (FS, 64, 64, 64, [140, 260], 3, 129, 0),
    (FS, 64, 64, 128, [140, 260], 3, 131, 33),
    (FS, 32, 32, 128, [161], 3, 131, 33),
    (BF, 64, 32, 128, [150], 3, 150, 0),         # 128
    (BF, 64, 32, 64, [150], 3, 150, 0),
    (FH, 60, 30, 128, [129, 5], 3, 2 ** 31 - 1, 0),
]


@pytest.mark.parametrize("case", CASES, ids=lambda c: "%s_%d_%d_d%d_n%s_w%d_win%d_s%d" % (str(c[0])[6:], c[1], c[2], c[3], "_".join(map(str, c[4])), *c[5:]))
def test_prompts_against_64_bits(case):
    dtype, h_q, h, d, lens, w, window, sinks = case
    print(case, flush=True)
    layer = layer_of(dtype, h_q, h, d, lens, w)
    q, K, V = inputs(dtype, h_q, h, d, sum(lens))
    out, lse = adakv.window_attn(layer, q, K, V, window, sinks, want_lse=True)
    torch.cuda.synchronize()
    check(layer, q, K, V, window, sinks, out, lse, heads=None if h_q < 16 else (0, 1, h_q // 2, h_q - 1))


# fp32: rows shared by one, two and four wavefronts (by the number of workgroups and what the rows see)
FP32_CASES = [
    (FS, 2, 1, 128, [3, 129, 257], 2, 2 ** 31 - 1, 0),
    (FS, 3, 3, 128, [700], 32, 2 ** 31 - 1, 0),
    (FS, 3, 3, 64, [700, 640], 32, 300, 40),
    (FS, 2, 2, 128, [900], 5, 65, 200),
    (FS, 16, 4, 128, [600, 130, 2], 1, 120, 1),
    (FS, 48, 6, 128, [500], 9, 2 ** 31 - 1, 0),
    (FS, 40, 10, 128, [40, 64, 33], 1, 64, 0),
    (FS, 64, 8, 128, [500, 400], 3, 50, 3),
    (FS, 64, 8, 64, [500, 400, 390], 3, 100, 3),
]


@pytest.mark.parametrize("case", FP32_CASES, ids=lambda c: "%d_%d_d%d_n%s_w%d_win%d_s%d" % (c[1], c[2], c[3], "_".join(map(str, c[4])), *c[5:]))
def test_fp32_prompts_against_64_bits(case):
    test_prompts_against_64_bits(case)


@pytest.mark.parametrize("dtype,d", [(BF, 128), (FH, 64), (FS, 64)])
def test_strided_tensors_loose_sequences_and_a_scale(dtype, d):
    """q, K and V as views into one fused buffer, NaN rows between the sequences, `out` rows of no sequence as they were."""
    print(dtype, d, flush=True)
    h_q, h, w, lens, gap = 4, 2, 4, [90, 131], 5
    off = [3, 3 + lens[0] + gap, 3 + lens[0] + gap + lens[1]]
    fused = torch.full((off[-1] + 2, h_q + 2 * h, d + 16), float("nan"), dtype=dtype, device=DEV)
    q, K, V = fused[:, :h_q, :d], fused[:, h_q:h_q + h, :d], fused[:, h_q + h:, :d]
    for b, n in enumerate(lens):
        for t, x in zip((q, K, V), inputs(dtype, h_q, h, d, n, seed=b)):
            t[off[b]:off[b] + n] = x
    strides = (fused.stride(0), fused.stride(1))
    layer = layer_of(dtype, h_q, h, d, lens, w, tok_off=off, scale=0.21, k_strides=strides, v_strides=strides)
    out = torch.full((off[-1] + 2, h_q, d), 7.0, dtype=dtype, device=DEV)
    row_lse = torch.full((2, h_q, w), 7.0, device=DEV)
    adakv.window_attn(layer, q, K, V, 50, 2, out=out, row_lse=row_lse)
    torch.cuda.synchronize()
    check(layer, q, K, V, 50, 2, out, row_lse)
    rest = torch.ones(len(out), dtype=torch.bool)
    for b, n in enumerate(lens):
        rest[off[b]:off[b] + n] = False
    assert (out[rest.to(DEV)] == 7.0).all()


@pytest.mark.parametrize("dtype,d", [(BF, 128), (FH, 128), (FS, 64)])
@pytest.mark.parametrize("what", [float("inf"), float("-inf"), float("nan")])
@pytest.mark.parametrize("window", [40, 130])
@pytest.mark.parametrize("h_q", [2, 70])
def test_hidden_keys_and_values_have_no_part(dtype, d, what, window, h_q):
    """Rows before a broken key or value, and rows whose window has left it behind, come out as if it were not there; the
    rows that see a broken value are not finite."""
    print(dtype, d, what, window, h_q, flush=True)
    n, w, sinks, at = 260, 4, 2, 101
    layer = layer_of(dtype, h_q, 1, d, [n], w)
    q, K, V = inputs(dtype, h_q, 1, d, n)
    clean = adakv.window_attn(layer, q, K, V, window, sinks)
    Vb, Kb = V.clone(), K.clone()
    Vb[at] = what
    Kb[at] = float("nan")
    sees = torch.zeros(n, dtype=torch.bool, device=DEV)
    sees[at:at + window] = True
    for K1, V1 in ((K, Vb), (Kb, V)):
        got = adakv.window_attn(layer, q, K1, V1, window, sinks)
        torch.cuda.synchronize()
        assert not torch.isfinite(got[sees].float()).any()
        check_rows = torch.nonzero(~sees)[:, 0].tolist()
        for hq in range(2):
            ref, lse, mag, big = S.prompt(f64(q[:, hq]), f64(K[:, 0]), f64(V[:, 0]), window, sinks, 1 / math.sqrt(d))
            keys = np.array([S.visible(i, n, window, sinks).sum() for i in range(n)])
            bound = attention_bound(dtype, d, ref, mag, big, lse, keys, rounded=True)
            assert_within(f64(got[:, hq])[check_rows], ref[check_rows], bound[check_rows], f"head {hq}")
    assert torch.isfinite(clean.float()).all()


@pytest.mark.parametrize("what", [float("inf"), float("nan")])
@pytest.mark.parametrize("window", [40, 230])
def test_hidden_values_in_fp32_rows_of_128(what, window):
    """As above, where four wavefronts share rows and a tile has no second place to be loaded to."""
    test_hidden_keys_and_values_have_no_part(FS, 128, what, window, 2)


def test_logits_far_apart_and_growing_along_the_keys():
    """The reference of the weights moves along a sequence: keys whose logits rise by hundreds, and fall again."""
    n, d, w = 400, 64, 4
    layer = layer_of(BF, 1, 1, d, [n], w, scale=1.0)
    q, K, V = inputs(BF, 1, 1, d, n, by=1.0)
    ramp = torch.cat([torch.linspace(-60, 60, 200), torch.linspace(60, -200, 200)]).to(DEV)
    q[:, 0, 0], K[:, 0, 0] = 8.0, ramp.to(BF)
    out, lse = adakv.window_attn(layer, q, K, V, n, want_lse=True)
    torch.cuda.synchronize()
    check(layer, q, K, V, n, 0, out, lse)


def test_row_lse_is_what_the_scoring_call_takes():
    """Scores from the call's log-sum-exp equal scores from one made in 64 bits, within what both may be off."""
    from paper_2407_11550_amd import synth
    wl = synth.small_workload(8, 2, 128, 16, 7, [700, 300], [2 * 90, 2 * 60], seed=5)
    q, K, V = synth.generate(wl, device=DEV)
    layer = adakv.Layer.from_workload(wl)
    qs = torch.zeros((wl.tok_off[-1], 8, 128), dtype=BF, device=DEV)
    for b, n in enumerate(wl.n):
        qs[wl.tok_off[b] + n:wl.tok_off[b + 1]] = q[b].transpose(0, 1)
    _, lse = adakv.window_attn(layer, qs, K, V, 4096, want_lse=True)
    want = synth.prefill_row_lse(wl, q, K)
    a, b = adakv.score(layer, q, K, row_lse=lse), adakv.score(layer, q, K, row_lse=want)
    torch.cuda.synchronize()
    off = float((lse - want).abs().max())
    assert off < 2e-5, off                       # (both in fp32: logits up to some 40, 128 products each)
    assert torch.allclose(a, b, rtol=2 * off + 1e-6, atol=0)


def test_what_lds_holds_before_a_call_has_no_part():
    """Short prompts right after calls that fill every compute unit's LDS with NaN: the result is that of a call after zeros."""
    layer = layer_of(BF, 8, 2, 128, [150, 20, 33], 8)
    q, K, V = inputs(BF, 8, 2, 128, 203)
    big = layer_of(BF, 32, 8, 128, [2048], 8)
    x = inputs(BF, 32, 8, 128, 2048)
    results = []
    for fill in (0.0, float("nan"), float("inf")):
        junk = torch.full_like(x[2], fill)
        adakv.window_attn(big, x[0], x[1], junk, 64)
        results.append(adakv.window_attn(layer, q, K, V, 70, 3))
        torch.cuda.synchronize()
    assert torch.equal(results[0], results[1]) and torch.equal(results[0], results[2])


def test_the_same_result_again_on_another_stream_and_from_a_graph():
    layer = layer_of(BF, 8, 2, 128, [700, 130], 32)
    q, K, V = inputs(BF, 8, 2, 128, 830)
    want, lse = adakv.window_attn(layer, q, K, V, 200, 4, want_lse=True)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    for _ in range(5):                           # (an `out` made by the call is cleared on the stream that the call runs on)
        got = adakv.window_attn(layer, q, K, V, 200, 4, stream=side)
        side.synchronize()
        assert torch.equal(got, want)
    out, row_lse = torch.zeros_like(want), torch.zeros_like(lse)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        adakv.window_attn(layer, q, K, V, 200, 4, out=out, row_lse=row_lse)
    for i in range(3):
        out.fill_(float(i))
        row_lse.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want) and torch.equal(row_lse, lse)
        adakv.window_attn(layer, q, K, V, 200, 4)
    again = adakv.window_attn(layer, q * 2, K, V, 200, 4)
    q.copy_(q * 2)
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(out, again)

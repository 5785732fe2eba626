"""Decoding steps over a window and sinks of a flattened cache against 64 bits."""
import math

import numpy as np
import pytest
import torch

import paper_2407_11550_amd as adakv
from oracle import decode_oracle as D
from oracle import serve_oracle as S
from serve_util import DEV, assert_within, attention_bound, f64, lse_bound, offsets

pytestmark = pytest.mark.gpu
BF, FH, FS = torch.bfloat16, torch.float16, torch.float32


def cache(dtype, g, h, d, lens, headroom, w=1, seed=0):
    """A layer whose segments hold lens rows, with head-room; spare rows are NaN."""
    gen = torch.Generator().manual_seed(seed)
    batch, cu = len(lens) // h, offsets(lens)
    per = [lens[b * h:(b + 1) * h] for b in range(batch)]
    layer = adakv.Layer(dtype, g * h, h, d, w, 7, 0.2, [max(p) for p in per], [sum(p) for p in per])
    rows = int(cu[-1]) + len(lens) * headroom
    K, V = (torch.full((rows, d), float("nan"), dtype=dtype, device=DEV) for _ in range(2))
    for s, a in enumerate(D.segment_starts(cu, headroom)):
        for t in (K, V):
            t[a:a + lens[s]] = torch.randn((lens[s], d), generator=gen).to(dtype).to(DEV)
    q, kn, vn = ((torch.randn((batch, k, d), generator=gen) * f).to(dtype).to(DEV) for k, f in ((g * h, 2.0), (h, 1.0), (h, 1.0)))
    return (layer, K, V, torch.tensor(cu, dtype=torch.int32, device=DEV), torch.tensor(lens, dtype=torch.int32, device=DEV), q, kn, vn)


def check(layer, q, K, V, cu, headroom, lens, window, sinks, out, lse, what=""):
    h, g, d = layer.h_kv, layer.h_q // layer.h_kv, layer.d
    start = D.segment_starts(cu.cpu().numpy(), headroom)
    for s, n in enumerate(lens):
        b, c = s // h, s % h
        got, got_lse = f64(out[b, c * g:(c + 1) * g]), f64(lse[b, c * g:(c + 1) * g])
        if n == 0:
            assert not got.any() and np.isneginf(got_lse).all(), what
            continue
        see = start[s] + S.step_rows(int(n), window, sinks)
        Ks, Vs = f64(K[torch.as_tensor(see, device=DEV)]), f64(V[torch.as_tensor(see, device=DEV)])
        for i in range(g):
            ref, z, mag, big = S.attend(f64(q[b, c * g + i]), Ks, Vs, layer.scale or 1 / math.sqrt(d))
            keys = np.array(len(see))
            assert_within(got[i], ref, attention_bound(layer.torch_dtype, d, ref, mag, np.array(big), np.array(z), keys, rounded=False), f"{what} segment {s}")
            assert_within(got_lse[i], z, lse_bound(d, np.array(big), np.array(z), keys), f"{what} lse {s}")


CASES = [
    # dtype g  h  d    lengths                          headroom window sinks
    (BF, 4, 2, 128, [300, 900, 33, 1200], 3, 100, 4),
    (BF, 4, 2, 128, [300, 900, 33, 1200], 3, 1, 0),
    (BF, 8, 1, 128, [2500], 5, 700, 37),          # in parts
    (BF, 8, 1, 64, [2500, 90], 5, 64, 64),
    (BF, 1, 3, 128, [700, 1, 66], 2, 50, 1),      # the vector kernel
    (BF, 2, 2, 64, [64, 65], 1, 32, 32),
    (FH, 4, 2, 64, [500, 31], 4, 129, 3),
    (FH, 2, 2, 128, [500, 310], 4, 129, 33),
    (FH, 1, 1, 128, [900], 4, 2 ** 31 - 1, 0),    # all of it
    (FS, 1, 2, 64, [400, 2], 3, 77, 5),
    (FS, 4, 1, 128, [1000], 3, 200, 130),
    (FS, 8, 1, 128, [333], 0, 40, 2 ** 31 - 1),
    (BF, 4, 70, 64, [40 + 7 * (i % 9) for i in range(70)], 2, 20, 3),    # more segments than lanes
]


@pytest.mark.parametrize("case", CASES, ids=lambda c: "%s_g%d_h%d_d%d_n%d_win%d_s%d" % (str(c[0])[6:], c[1], c[2], c[3], c[4][0], c[6], c[7]))
def test_attention_and_steps_against_64_bits(case):
    dtype, g, h, d, lens, hr, window, sinks = case
    print(case, flush=True)
    if h > 64:
        lens, h = lens * 2, 35                    # two heads' worth per sequence: four sequences
    layer, K, V, cu, seg_len, q, kn, vn = cache(dtype, g, h, d, lens, hr)
    out, lse = adakv.decode_attn(layer, q, cu, hr, K, V, seg_len, want_lse=True, window=window, sinks=sinks)
    torch.cuda.synchronize()
    check(layer, q, K, V, cu, hr, lens, window, sinks, out, lse, "attention")
    over = torch.zeros(1, dtype=torch.int32, device=DEV)
    held = np.array(lens)
    for t in range(hr + 1):
        before = (K.clone(), V.clone())
        out, lse = adakv.decode_step(layer, q, kn, vn, cu, hr, K, V, seg_len, overflow=over, want_lse=True, window=window, sinks=sinks)
        torch.cuda.synchronize()
        if t < hr:
            at = torch.as_tensor(D.segment_starts(cu.cpu().numpy(), hr) + held, device=DEV)
            before[0][at], before[1][at] = kn.view(-1, d), vn.view(-1, d)
            held = held + 1
        for was, now in zip(before, (K, V)):
            assert torch.equal(was.view(torch.uint8), now.view(torch.uint8))
        assert np.array_equal(seg_len.cpu().numpy(), held) and int(over) == (t >= hr)
        if t in (0, hr):
            check(layer, q, K, V, cu, hr, held, window, sinks, out, lse, f"step {t}")


@pytest.mark.parametrize("lens, window, kernels", [([900, 61], 100, 1), ([2500, 61], 1500, 2)], ids=["one_workgroup", "parts"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("g", [1, 2, 4, 8])
@pytest.mark.parametrize("dtype", [BF, FH, FS])
def test_a_segment_by_one_workgroup_and_in_parts(dtype, g, d, lens, window, kernels):
    """Both divisions of the work, for every kernel there is; the last step finds no room."""
    layer, K, V, cu, seg_len, q, kn, vn = cache(dtype, g, 2, d, lens, 1)
    over = torch.zeros(1, dtype=torch.int32, device=DEV)
    for t in range(2):
        trace = adakv.KernelTrace(8)
        with trace:
            out, lse = adakv.decode_step(layer, q, kn, vn, cu, 1, K, V, seg_len, overflow=over, want_lse=True, window=window, sinks=3)
        torch.cuda.synchronize()
        assert len(trace.durations_us()) == kernels
        held = np.array(lens) + 1
        assert np.array_equal(seg_len.cpu().numpy(), held) and int(over) == t
        check(layer, q, K, V, cu, 1, held, window, 3, out, lse, f"step {t}")


@pytest.mark.parametrize("dtype", [BF, FS])
def test_many_segments_that_hold_their_window(dtype):
    lens = [1010 + i % 5 for i in range(256)]
    layer, K, V, cu, seg_len, q, _, _ = cache(dtype, 4, 32, 128, lens, 2)
    trace = adakv.KernelTrace(8)
    with trace:
        out, lse = adakv.decode_attn(layer, q, cu, 2, K, V, seg_len, want_lse=True, window=1000, sinks=4)
    torch.cuda.synchronize()
    assert len(trace.durations_us()) == 1
    check(layer, q, K, V, cu, 2, np.array(lens), 1000, 4, out, lse)


@pytest.mark.parametrize("dtype", [BF, FH, FS])
def test_hidden_rows_have_no_part(dtype):
    layer, K, V, cu, seg_len, q, _, _ = cache(dtype, 4, 2, 64, [500, 260], 3)
    want = adakv.decode_attn(layer, q, cu, 3, K, V, seg_len, window=70, sinks=5)
    for s, a in enumerate((0, 503)):
        K[a + 5:a + (430, 190)[s]] = float("nan")
        V[a + 5:a + (430, 190)[s]] = float("inf")
    got = adakv.decode_attn(layer, q, cu, 3, K, V, seg_len, window=70, sinks=5)
    torch.cuda.synchronize()
    assert torch.equal(got, want) and torch.isfinite(got).all()


@pytest.mark.parametrize("lens, window", [([900, 61], 100), ([2500, 61], 1500)], ids=["one_workgroup", "parts"])
@pytest.mark.parametrize("dtype, g, d", [(BF, 4, 128), (BF, 1, 64), (FH, 8, 64), (FS, 4, 128)])
@pytest.mark.parametrize("what", [float("nan"), float("inf")])
def test_a_key_that_is_no_number_is_not_passed_over(dtype, g, d, lens, window, what):
    """A visible row of NaN or infinite keys, as the last appended one: the group's results are no numbers, the others are."""
    layer, K, V, cu, seg_len, q, _, _ = cache(dtype, g, 2, d, lens, 3)
    K[lens[0] - 1] = what
    out, lse = adakv.decode_attn(layer, q.abs() + 1.0, cu, 3, K, V, seg_len, want_lse=True, window=window, sinks=2)
    torch.cuda.synchronize()
    assert torch.isnan(out[0, :g]).all() and torch.isnan(lse[0, :g]).all()
    assert torch.isfinite(out[0, g:]).all() and torch.isfinite(lse[0, g:]).all()


def test_empty_and_corrupt_lengths():
    layer, K, V, cu, seg_len, q, kn, vn = cache(BF, 4, 3, 128, [60, 50, 40], 3)
    seg_len[1] = 0
    out, lse = adakv.decode_attn(layer, q, cu, 3, K, V, seg_len, want_lse=True, window=7, sinks=1)
    torch.cuda.synchronize()
    check(layer, q, K, V, cu, 3, [60, 0, 40], 7, 1, out, lse)
    out = adakv.decode_step(layer, q, kn, vn, cu, 3, K, V, seg_len, window=1)
    torch.cuda.synchronize()
    assert seg_len.tolist() == [61, 1, 41]
    # a window of one row sees the appended one alone
    assert torch.equal(out.view(3, 4, 128), vn.float().view(3, 1, 128).expand(3, 4, 128))


def test_a_window_as_long_as_the_cache_is_no_window():
    layer, K, V, cu, seg_len, q, _, _ = cache(BF, 4, 8, 128, [900, 20, 1500, 64, 65, 7, 300, 301], 4)
    a = adakv.decode_attn(layer, q, cu, 4, K, V, seg_len)
    b = adakv.decode_attn(layer, q, cu, 4, K, V, seg_len, window=5000)
    torch.cuda.synchronize()
    assert torch.equal(a, b)


def test_a_captured_step():
    layer, K, V, cu, seg_len, q, kn, vn = cache(BF, 4, 2, 128, [600, 40], 8)
    ref = [t.clone() for t in (K, V, seg_len)]
    ws = torch.empty(adakv.decode_workspace_bytes(layer, 8), dtype=torch.uint8, device=DEV)
    out, lse = torch.zeros((1, 8, 128), device=DEV), torch.zeros((1, 8), device=DEV)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        adakv.decode_step(layer, q, kn, vn, cu, 8, K, V, seg_len, out=out, lse=lse, ws=ws, window=33, sinks=2)
    for _ in range(3):
        graph.replay()
        want = adakv.decode_step(layer, q, kn, vn, cu, 8, *ref, window=33, sinks=2)
        torch.cuda.synchronize()
        assert torch.equal(out, want) and torch.equal(seg_len, ref[2])

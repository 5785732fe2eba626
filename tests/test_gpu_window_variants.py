"""Every kernel of prompt attention, by the name that the trace gives it (one, two or four wavefronts share 32 rows), over
several tiles of keys: tiles skipped between sinks and window, a reference that moves, a value that is no number."""
import math

import numpy as np
import pytest
import torch

import paper_2407_11550_amd as adakv
from oracle import serve_oracle as S
from serve_util import DEV, assert_within, attention_bound, f64, lse_bound

pytestmark = pytest.mark.gpu
BF, FH, FS = torch.bfloat16, torch.float16, torch.float32
NAMES = {1: "window_attn", 2: "window_attn_2", 4: "window_attn_4"}

# (type, d, wavefronts that share rows) -> query heads, lengths: sequences with four tiles at least, of 32 or 64 keys where
# rows are not shared, of as many times 32 as wavefronts share them
SHAPES = {
    (BF, 64, 1): (64, [700, 290, 129]), (BF, 64, 2): (64, [300]), (BF, 64, 4): (8, [700, 65]),
    (BF, 128, 1): (64, [530, 290]), (BF, 128, 2): (64, [290]), (BF, 128, 4): (8, [700, 65]),
    (FS, 64, 1): (64, [700, 650, 300]), (FS, 64, 2): (64, [300]), (FS, 64, 4): (8, [700, 65]),
    (FS, 128, 1): (64, [530, 290]), (FS, 128, 2): (64, [290]), (FS, 128, 4): (8, [700, 65]),
}
SHAPES.update({(FH,) + k[1:]: v for k, v in SHAPES.items() if k[0] == BF})
KINDS = sorted(SHAPES, key=str)
kinds = pytest.mark.parametrize("kind", KINDS, ids=lambda k: "%s_d%d_share%d" % (str(k[0])[6:], *k[1:]))
W = 5


def make(kind, by=2.0):
    dtype, d, _ = kind
    h_q, lens = SHAPES[kind]
    layer = adakv.Layer(dtype, h_q, 2, d, W, 7, 0.2, [n - W for n in lens], [2 * W for _ in lens])
    g = torch.Generator().manual_seed(d + h_q)
    return layer, *((torch.randn((sum(lens), k, d), generator=g) * f).to(dtype).to(DEV) for k, f in ((h_q, by), (2, 1.0), (2, 1.0)))


def call(kind, layer, q, K, V, window, sinks):
    trace = adakv.KernelTrace(4)
    with trace:
        out, lse = adakv.window_attn(layer, q, K, V, window, sinks, want_lse=True)
    torch.cuda.synchronize()
    assert [name for name, _ in trace.durations_us()] == [NAMES[kind[2]]], kind
    return out, lse


def check(layer, q, K, V, window, sinks, out, lse, heads, skip=None):
    """Against 64 bits; of each sequence but the rows that `skip` says."""
    d, g = layer.d, layer.h_q // layer.h_kv
    for b in range(layer.batch):
        n, t0 = layer.n[b] + W, layer.tok_off[b]
        rows = np.array([i for i in range(n) if skip is None or not skip(i, n)])
        keys = np.array([S.visible(i, n, window, sinks).sum() for i in range(n)])
        for hq in heads:
            ref, z, mag, big = S.prompt(f64(q[t0:t0 + n, hq]), f64(K[t0:t0 + n, hq // g]), f64(V[t0:t0 + n, hq // g]), window, sinks, 1 / math.sqrt(d))
            bound = attention_bound(layer.torch_dtype, d, ref, mag, big, z, keys, rounded=True)
            assert_within(f64(out[t0:t0 + n, hq])[rows], ref[rows], bound[rows], f"sequence {b} head {hq}")
            assert_within(f64(lse[b, hq]), z[n - W:], lse_bound(d, big, z, keys)[n - W:], f"lse {b} {hq}")


@kinds
@pytest.mark.parametrize("window, sinks", [(10 ** 6, 0), (100, 35)])
def test_every_kernel_over_several_tiles(kind, window, sinks):
    print(kind, window, sinks, flush=True)
    layer, q, K, V = make(kind)
    out, lse = call(kind, layer, q, K, V, window, sinks)
    check(layer, q, K, V, window, sinks, out, lse, (0, layer.h_q - 1))


@kinds
def test_a_reference_that_moves(kind):
    """Logits that rise by some 100 along the keys and fall again: weights are taken against one reference after another."""
    print(kind, flush=True)
    layer, q, K, V = make(kind, by=1.0)
    for b in range(layer.batch):
        n, t0 = layer.n[b] + W, layer.tok_off[b]
        ramp = 50.0 - 100.0 * (torch.arange(n, device=DEV) / (0.6 * n) - 1.0).abs()
        K[t0:t0 + n, :, 0] = ramp.to(K.dtype)[:, None]
    q[:, :, 0] = math.sqrt(layer.d)
    out, lse = call(kind, layer, q, K, V, 10 ** 6, 0)
    check(layer, q, K, V, 10 ** 6, 0, out, lse, (0, layer.h_q - 1))


@kinds
@pytest.mark.parametrize("what", [float("nan"), float("inf")])
def test_a_value_that_is_hidden_from_most_rows(kind, what):
    print(kind, what, flush=True)
    layer, q, K, V = make(kind)
    window, sinks, at = 100, 35, 52
    broken = V.clone()
    for b in range(layer.batch):
        broken[layer.tok_off[b] + at] = what
    out, lse = call(kind, layer, q, K, broken, window, sinks)
    sees = lambda i, n: at <= i < at + window
    check(layer, q, K, V, window, sinks, out, lse, (0, layer.h_q - 1), skip=sees)
    for b in range(layer.batch):
        n, t0 = layer.n[b] + W, layer.tok_off[b]
        rows = [t0 + i for i in range(n) if sees(i, n)]
        assert not torch.isfinite(out[rows].float()).any()

"""Sequences of a cache forked, dropped and given other head-room, in every row width and in 8 bits; and the whole life of a
served cache in one piece."""
import numpy as np
import pytest
import torch

import paper_2407_11550_amd as adakv
from oracle import adakv_oracle as O
from oracle import serve_oracle as S
from paper_2407_11550_amd import synth
from serve_util import DEV, offsets

pytestmark = pytest.mark.gpu
BF, FH, FS = torch.bfloat16, torch.float16, torch.float32


def source(dtype, h, d, lens, headroom, held, q8):
    per = [lens[b * h:(b + 1) * h] for b in range(len(lens) // h)]
    layer = adakv.Layer(dtype, h, h, d, 1, 7, 0.2, [max(p) for p in per], [sum(p) for p in per])
    g = torch.Generator(device=DEV).manual_seed(5)
    rows = adakv.cache_rows(layer, headroom)
    if q8:
        cache = adakv.q8_cache(layer, headroom, DEV)
        for t in cache[:2]:
            t.view(torch.uint8).copy_(torch.randint(0, 127, t.shape, generator=g, device=DEV, dtype=torch.uint8))
        for t in cache[2:]:
            t.copy_(torch.rand(t.shape, generator=g, device=DEV))
    else:
        cache = [torch.randn((rows, d), generator=g, device=DEV).to(dtype) for _ in range(2)]
    return layer, cache, torch.tensor(offsets(lens), dtype=torch.int32, device=DEV), torch.tensor(held, dtype=torch.int32, device=DEV)


CASES = [
    # h  lengths at the start       headroom  held                    picks            new head-room
    (2, [5, 9, 40, 3], 7, [6, 9, 47, 0], [1, 0, 1, 1], 7),
    (1, [300], 0, [300], [0] * 64, 3),
    (3, [33, 1, 64, 32, 31, 65, 2, 200, 7], 33, [66, 34, 64, 32, 31, 98, 35, 233, 40], [2, 0], 100),
    (2, [20, 20, 50, 8], 30, [50, 20, 60, 9], [1, 0], 4),            # too little room for some
    (64, [1 + i % 5 for i in range(128)], 2, [2 + i % 5 for i in range(128)], [1], 0),
]


@pytest.mark.parametrize("dtype,d,q8", [(BF, 64, False), (FH, 128, False), (FS, 128, False), (FS, 64, True), (BF, 128, True)])
@pytest.mark.parametrize("case", CASES, ids=lambda c: "h%d_n%d_to%d_hr%d" % (c[0], c[1][0], len(c[4]), c[5]))
def test_moved_rows_scales_lengths_and_offsets(case, dtype, d, q8):
    h, lens, hr, held, picks, new = case
    print(case, dtype, d, q8, flush=True)
    layer, cache, cu, seg_len = source(dtype, h, d, lens, hr, held, q8)
    cu_out, lens_out, runs, over = S.move(picks, h, cu.cpu().numpy(), hr, held, new)
    overflow = torch.zeros(1, dtype=torch.int32, device=DEV)
    to = layer.pick(picks)
    if q8:
        out = adakv.q8_cache(to, new, DEV)
        for t in out:
            t.view(torch.uint8).fill_(0x55)
        to, cu_got, out, len_got = adakv.cache_move_q8(layer, picks, cu, hr, cache, seg_len, new, out=out, overflow=overflow)
    else:
        out = [torch.full((adakv.cache_rows(to, new), d), 9.0, dtype=dtype, device=DEV) for _ in range(2)]
        to, cu_got, *out, len_got = adakv.cache_move(layer, picks, cu, hr, *cache, seg_len, new, K_out=out[0], V_out=out[1], overflow=overflow)
    torch.cuda.synchronize()
    assert np.array_equal(cu_got.cpu().numpy(), cu_out) and np.array_equal(len_got.cpu().numpy(), lens_out) and bool(overflow) == over
    assert to.batch == len(picks) and to.num_rows_out == cu_out[-1]
    untouched = out[0].view(torch.uint8).flatten()[:1].tolist()
    for src, dst in zip(cache[:2], out[:2]):
        want = torch.full_like(dst.view(torch.uint8), 0x55) if q8 else torch.full_like(dst, 9.0)
        for a, b, n in runs:
            want[b:b + n] = src.view(want.dtype)[a:a + n] if q8 else src[a:a + n]
        assert torch.equal(dst.view(want.dtype), want), untouched
    if q8:
        p_in, p_out = S.scale_places(cu.cpu().numpy(), hr), S.scale_places(cu_out, new)
        segs = [b * h + c for b in picks for c in range(h)]
        for src, dst in zip(cache[2:], out[2:]):
            want = torch.full_like(dst.view(torch.uint8), 0x55).view(torch.float32)
            for i, (s, n) in enumerate(zip(segs, lens_out)):
                k = -(-int(n) // S.BLOCK)
                want[p_out[i]:p_out[i] + k] = src[p_in[s]:p_in[s] + k]
            assert torch.equal(dst.view(torch.int32), want.view(torch.int32))


def test_corrupt_lengths_stay_inside():
    """Lengths below zero and beyond the capacity are taken as none and as full."""
    layer, cache, cu, seg_len = source(BF, 2, 64, [10, 20], 3, [-5, 1 << 20], False)
    _, _, K, V, lens = adakv.cache_move(layer, [0], cu, 3, *cache, seg_len, 3)
    torch.cuda.synchronize()
    assert lens.tolist() == [0, 23]
    assert torch.equal(K[13:36], cache[0][13:36]) and not K[:13].any() and torch.equal(V[13:36], cache[1][13:36])


def test_source_and_destination_may_not_overlap(lib):
    layer, cache, cu, seg_len = source(BF, 2, 64, [10, 20], 3, [10, 20], False)
    for kw in (dict(K_out=cache[0]), dict(V_out=cache[1]), dict(len_out=seg_len), dict(cu_out=cu), dict(K_out=cache[1])):
        with pytest.raises(adakv.AdaKVError, match="invalid"):
            adakv.cache_move(layer, [0], cu, 3, *cache, seg_len, 3, **kw)


@pytest.mark.parametrize("q8", [False, True])
def test_a_served_cache_from_prompt_to_forks(q8):
    """Prompt attention hands its log-sum-exp to the compression, its cache takes tokens until a head-room is used up, the
    batch is forked, thinned and given room, and both branches go on: the forks as the original would have."""
    wl = synth.small_workload(8, 2, 128, 16, 7, [900, 400], [2 * 150, 2 * 90], seed=11)
    q, K, V = synth.generate(wl, device=DEV)
    layer = adakv.Layer.from_workload(wl)
    qs = torch.randn((wl.tok_off[-1], 8, 128), device=DEV).to(BF)
    for b, n in enumerate(wl.n):
        qs[wl.tok_off[b] + n:wl.tok_off[b + 1]] = q[b].transpose(0, 1)
    _, lse = adakv.window_attn(layer, qs, K, V, 1 << 20, want_lse=True)
    res = adakv.compress(layer, q, K, V, row_lse=lse)
    torch.cuda.synchronize()
    for b in range(2):                           # the eviction decision follows the scores
        sc = res["scores"][2 * sum(wl.n[:b]):2 * sum(wl.n[:b + 1])].view(2, -1).cpu().numpy()
        bud, _ = O.allocate(sc, wl.B[b], wl.w, wl.alpha)
        assert np.array_equal(res["budgets"][2 * b:2 * b + 2].cpu().numpy(), bud)
    hr, cu = 3, res["cu_seqlens"]
    if q8:
        cache, seg_len = adakv.cache_build_q8(layer, K, V, res["indices"], cu, hr)
    else:
        *cache, seg_len = adakv.cache_build(layer, K, V, res["indices"], cu, hr)

    def step(lay, t, cu, hr, cache, seg_len, over, rows):
        x = torch.Generator(device=DEV).manual_seed(100 + t)
        q, k, v = (torch.randn((2, n, 128), generator=x, device=DEV).to(BF)[rows].contiguous() for n in (8, 2, 2))
        if q8:
            return adakv.decode_step_q8(lay, q, k, v, cu, hr, cache, seg_len, overflow=over)
        return adakv.decode_step(lay, q, k, v, cu, hr, *cache, seg_len, overflow=over)

    over = torch.zeros(1, dtype=torch.int32, device=DEV)
    for t in range(hr):
        step(layer, t, cu, hr, cache, seg_len, over, [0, 1])
    picks = [1, 0, 1]
    if q8:
        to, cu2, cache2, len2 = adakv.cache_move_q8(layer, picks, cu, hr, cache, seg_len, 20)
        big, cu3, cache3, len3 = adakv.cache_move_q8(layer, [0, 1], cu, hr, cache, seg_len, 20)
    else:
        to, cu2, *cache2, len2 = adakv.cache_move(layer, picks, cu, hr, *cache, seg_len, 20)
        big, cu3, *cache3, len3 = adakv.cache_move(layer, [0, 1], cu, hr, *cache, seg_len, 20)
    for t in range(hr, hr + 5):
        a = step(to, t, cu2, 20, cache2, len2, over, picks)
        b = step(big, t, cu3, 20, cache3, len3, over, [0, 1])
        torch.cuda.synchronize()
        assert torch.allclose(a, b[picks], rtol=0, atol=2e-5 * float(b.abs().max()))     # (parts are cut differently: fp32 sums)
    assert int(over) == 0
    step(layer, 99, cu, hr, cache, seg_len, over, [0, 1])
    torch.cuda.synchronize()
    assert int(over) == 1

"""Decoding steps of sequences that share caches, against 64 bits."""
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


def cache(gen, dtype, h_q, h, d, lens, headroom, kept=None):
    """A layer whose segments hold `lens` rows of the `kept` they were built with and the head-room; spare rows are NaN."""
    kept = [max(1, n) for n in lens] if kept is None else kept
    cu = offsets(kept)
    per = [kept[b:b + h] for b in range(0, len(kept), h)]
    layer = adakv.Layer(dtype, h_q, h, d, 1, 7, 0.2, [max(p) for p in per], [sum(p) for p in per])
    rows = int(cu[-1]) + len(lens) * headroom
    K, V = (torch.full((rows, d), float("nan"), dtype=dtype, device=DEV) for _ in range(2))
    for s, a in enumerate(D.segment_starts(cu, headroom)):
        for t in (K, V):
            t[a:a + lens[s]] = torch.randn((lens[s], d), generator=gen).to(dtype).to(DEV)
    return layer, K, V, torch.tensor(cu, dtype=torch.int32, device=DEV), torch.tensor(lens, dtype=torch.int32, device=DEV)


class Case:
    def __init__(self, dtype, g, h, d, of, shared, own, headroom=3, shared_headroom=0, seed=0, q_by=2.0):
        gen = torch.Generator().manual_seed(seed)
        self.dtype, self.g, self.h, self.d, self.of, self.headroom, self.batch = dtype, g, h, d, of, headroom, len(of)
        self.shared, self.own, self.shared_headroom = list(shared), list(own), shared_headroom
        self.layer, self.K, self.V, self.cu, self.lens = cache(gen, dtype, g * h, h, d, self.own, headroom)
        self.p_layer, self.pK, self.pV, self.p_cu, self.p_lens = cache(gen, dtype, g * h, h, d, self.shared, shared_headroom)
        self.prefix = adakv.Prefix(self.p_layer, self.p_cu, shared_headroom, self.pK, self.pV, self.p_lens, of)
        self.q, self.k, self.v = ((torch.randn((self.batch, n, d), generator=gen) * f).to(dtype).to(DEV)
                                  for n, f in ((g * h, q_by), (h, 1.0), (h, 1.0)))

    def rows(self, s, n):
        """Keys and values that query heads of own segment s see, n of them its own."""
        b, c = s // self.h, s % self.h
        a = D.segment_starts(self.cu.cpu().numpy(), self.headroom)[s]
        parts = [(self.K[a:a + n], self.V[a:a + n])]
        if self.of[b] >= 0:
            t = self.of[b] * self.h + c
            a = D.segment_starts(self.p_cu.cpu().numpy(), self.shared_headroom)[t]
            parts.insert(0, (self.pK[a:a + self.shared[t]], self.pV[a:a + self.shared[t]]))
        return tuple(f64(torch.cat([p[i] for p in parts])) for i in range(2))

    def check(self, out, lse, held, what=""):
        """As for the other steps; a weight over a shared segment is 2^-23 off at most (three bf16 parts 2^-24, two fp16 parts 2^-22 / 2), and
        in fp16 2^-45 of the largest."""
        worst = [0.0, 0.0]
        for s in range(self.batch * self.h):
            b, c = s // self.h, s % self.h
            Ks, Vs = self.rows(s, int(held[s]))
            heads = slice(c * self.g, (c + 1) * self.g)
            got, got_lse = f64(out[b, heads]), f64(lse[b, heads])
            if len(Ks) == 0:
                assert not got.any() and np.isneginf(got_lse).all(), f"{what} segment {s}"
                continue
            assert np.isfinite(got).all() and np.isfinite(got_lse).all(), f"{what} segment {s}: not finite"
            for i in range(self.g):
                ref, z, mag, big = S.attend(f64(self.q[b, c * self.g + i]), Ks, Vs, self.layer.scale or 1 / math.sqrt(self.d))
                keys = np.array(len(Ks))
                bound = attention_bound(self.dtype, self.d, ref, mag, np.array(big), np.array(z), keys, rounded=False)
                if self.dtype != FS:
                    bound = bound + mag * 2.0 ** -23
                if self.dtype == FH:
                    bound = bound + len(Ks) * 2.0 ** -45 * np.abs(Vs).max()
                worst[0] = max(worst[0], float((np.abs(got[i] - ref) / bound).max()))
                worst[1] = max(worst[1], float(np.abs(got_lse[i] - z) / lse_bound(self.d, np.array(big), np.array(z), keys)))
        print(f"  {what}: errors at most {worst[0]:.3f} and {worst[1]:.3f} of their bounds", flush=True)
        assert worst[0] <= 1 and worst[1] <= 1, what

    def attn(self, **kw):
        return adakv.decode_prefix_attn(self.layer, self.q, self.cu, self.headroom, self.K, self.V, self.lens, self.prefix, want_lse=True, **kw)

    def step(self, **kw):
        return adakv.decode_prefix_step(self.layer, self.q, self.k, self.v, self.cu, self.headroom, self.K, self.V, self.lens, self.prefix,
                                        **dict(dict(want_lse=True), **kw))


def spread(rng, n, most):
    """n lengths up to most, at the places where tiles, wavefronts and parts end among them."""
    ends = [v for v in (0, 1, 31, 32, 33, 63, 64, 65, 127, 128, 129, 255, 257) if v <= most]
    return [int(rng.choice(ends)) if rng.random() < 0.5 else int(rng.integers(0, most + 1)) for _ in range(n)]


CASES = [
    # dtype g  h  d    sequences groups longest shared, own
    (BF, 4, 2, 128, 2, 1, 300, 40),             # 32 rows of queries a workgroup
    (BF, 8, 2, 128, 4, 1, 700, 70),
    (BF, 1, 3, 64, 5, 2, 500, 130),
    (BF, 2, 2, 64, 16, 1, 1000, 20),
    (BF, 8, 1, 128, 8, 1, 900, 300),            # 64
    (BF, 4, 2, 64, 13, 1, 900, 60),
    (BF, 8, 2, 128, 16, 1, 600, 30),            # 128
    (BF, 8, 1, 64, 12, 1, 1200, 30),
    (BF, 8, 1, 128, 64, 1, 900, 9),             # several blocks of rows
    (BF, 8, 2, 64, 50, 2, 700, 9),
    (FH, 4, 2, 128, 3, 1, 500, 90),
    (FH, 4, 2, 64, 3, 2, 500, 90),
    (FH, 8, 1, 128, 7, 1, 700, 33),
    (FH, 2, 2, 64, 30, 1, 600, 65),
    (FH, 8, 1, 128, 20, 1, 500, 20),
    (FH, 8, 1, 64, 33, 2, 500, 20),
    (FS, 4, 2, 128, 4, 1, 300, 50),
    (FS, 4, 2, 64, 4, 2, 300, 50),
    (FS, 8, 1, 128, 8, 1, 300, 20),
    (FS, 8, 1, 64, 7, 1, 300, 20),
    (FS, 8, 1, 128, 18, 1, 300, 20),
    (FS, 4, 1, 64, 41, 1, 300, 20),
]


@pytest.mark.parametrize("dtype,g,h,d,batch,groups,longest,own", CASES)
def test_attention_over_both(dtype, g, h, d, batch, groups, longest, own):
    rng = np.random.default_rng(batch * 100 + g)
    of = [int(p) for p in rng.integers(0, groups, size=batch)]
    shared = spread(rng, groups * h, longest)
    shared[0] = longest
    c = Case(dtype, g, h, d, of, shared, spread(rng, batch * h, own), shared_headroom=int(rng.integers(0, 5)))
    before = [t.clone() for t in (c.K, c.V, c.lens, c.pK, c.pV, c.p_lens)]
    out, lse = c.attn()
    c.check(out, lse, c.own, f"{dtype} g {g} d {d} batch {batch}")
    for t, was in zip((c.K, c.V, c.lens, c.pK, c.pV, c.p_lens), before):
        assert torch.equal(t.view(torch.uint8), was.view(torch.uint8))


@pytest.mark.parametrize("dtype,g,h,d,batch,groups,longest,own", CASES[::3])
def test_steps(dtype, g, h, d, batch, groups, longest, own):
    """Three tokens: rows appended as decode_step appends them, lengths that grow, a segment that is full in the third."""
    rng = np.random.default_rng(batch * 100 + g + 1)
    c = Case(dtype, g, h, d, [int(p) for p in rng.integers(-1, groups, size=batch)], spread(rng, groups * h, longest), [own] * (batch * h), headroom=2)
    overflow = torch.zeros(1, dtype=torch.int32, device=DEV)
    ws = torch.zeros(adakv.prefix_workspace_bytes(c.layer, 2, c.prefix), dtype=torch.uint8, device=DEV)
    for turn in range(3):
        K, V, lens = c.K.clone(), c.V.clone(), c.lens.clone()
        plain = torch.zeros(1, dtype=torch.int32, device=DEV)
        adakv.append(c.layer, c.k, c.v, c.cu, 2, K, V, lens, overflow=plain)
        out, lse = c.step(overflow=overflow, ws=ws)
        for t, want in ((c.K, K), (c.V, V), (c.lens, lens), (overflow, plain)):
            assert torch.equal(t.view(torch.uint8), want.view(torch.uint8)), turn
        c.check(out, lse, c.lens.cpu().numpy(), f"token {turn}")
        c.q, c.k, c.v = c.q.flip(0).contiguous(), (c.v * 0.5).contiguous(), (c.k * 2).contiguous()
    assert overflow.item() == 1


@pytest.mark.parametrize("dtype,d", [(BF, 128), (FH, 64), (FS, 64)])
def test_long_segments_in_parts(dtype, d):
    """Uneven heads of some thousand rows; one sequence without a shared cache, one shared cache without sequences."""
    rng = np.random.default_rng(5)
    of = [2, 0, -1, 0, 2, 0, 0]
    c = Case(dtype, 4, 2, d, of, [9000, 2500, 700, 800, 4097, 64], spread(rng, 14, 200), shared_headroom=7)
    out, lse = c.attn()
    c.check(out, lse, c.own, "long")


def test_more_segments_than_a_wavefront_has_lanes():
    rng = np.random.default_rng(6)
    of = [int(p) for p in rng.integers(0, 20, size=40)]
    c = Case(BF, 2, 7, 64, of, spread(rng, 140, 300), spread(rng, 280, 40))
    out, lse = c.attn()
    c.check(out, lse, c.own, "140 shared segments")


@pytest.mark.parametrize("dtype,d,groups,h", [(BF, 128, 3, 2), (FH, 64, 3, 2), (BF, 64, 9, 8), (FS, 64, 13, 5)])
def test_shared_caches_of_many_and_of_few(dtype, d, groups, h):
    """One cache for most sequences, whose query rows make several blocks, others for a few of them, one for none; up to 64 segments and more."""
    rng = np.random.default_rng(groups)
    of = [0] * 37 + [1] * 9 + ([int(p) for p in rng.integers(3, groups, size=10)] if groups > 3 else []) + [-1]
    c = Case(dtype, 8, h, d, of, spread(rng, groups * h, 900), spread(rng, len(of) * h, 20), shared_headroom=3)
    out, lse = c.attn()
    c.check(out, lse, c.own, f"{groups} shared caches, {h} heads")


@pytest.mark.parametrize("dtype,d,batch,name", [(BF, 128, 4, "prefix_attn_2"), (BF, 64, 4, "prefix_attn_4"), (FH, 128, 4, "prefix_attn_2"), (FH, 64, 4, "prefix_attn_4"),
                                                (FS, 128, 4, "prefix_attn_8"), (FS, 64, 3, "prefix_attn_8"), (FS, 128, 8, "prefix_attn_8"), (FS, 128, 9, "prefix_attn_2"),
                                                (FS, 64, 16, "prefix_attn_2"), (BF, 128, 16, "prefix_attn_2"), (BF, 64, 16, "prefix_attn_2"),
                                                (FH, 64, 16, "prefix_attn_2"), (BF, 128, 17, "prefix_attn"), (BF, 64, 40, "prefix_attn"), (FH, 128, 17, "prefix_attn"),
                                                (FH, 64, 33, "prefix_attn"), (FS, 128, 17, "prefix_attn"), (FS, 64, 20, "prefix_attn")])
def test_every_kernel_over_several_tiles(dtype, d, batch, name):
    """By its name; segments of many tiles, in parts of several, whose last tile has few rows."""
    c = Case(dtype, 4, 2, d, [0] * batch, [18001, 2000], [300] * (2 * batch))
    with adakv.KernelTrace(8) as trace:
        out, lse = c.attn()
    torch.cuda.synchronize()
    assert [n for n, _ in trace.durations_us()] == [name, "prefix_combine"]
    some = [0, 1, batch - 1]                   # (all query rows are alike in this: three sequences are looked at)
    for b in some:
        for h in range(2):
            s = b * 2 + h
            Ks, Vs = c.rows(s, 300)
            for i in range(4):
                ref, z, mag, big = S.attend(f64(c.q[b, 4 * h + i]), Ks, Vs, 1 / math.sqrt(d))
                keys = np.array(len(Ks))
                bound = attention_bound(dtype, d, ref, mag, np.array(big), np.array(z), keys, rounded=False) + (mag * 2.0 ** -23 if dtype != FS else 0.0)
                if dtype == FH:
                    bound = bound + len(Ks) * 2.0 ** -45 * np.abs(Vs).max()
                assert (np.abs(f64(out[b, 4 * h + i]) - ref) <= bound).all(), (b, h, i)
                assert abs(float(lse[b, 4 * h + i]) - z) <= lse_bound(d, np.array(big), np.array(z), keys), (b, h, i)


@pytest.mark.parametrize("dtype,d", [(t, d) for t in (BF, FH, FS) for d in (64, 128)])
def test_every_length_up_to_two_tiles(dtype, d):
    """64 sequences, each with a shared cache to itself: own lengths 0 to 127, shared ones 130 to 3."""
    c = Case(dtype, 4, 2, d, list(range(64)), [130 - n for n in range(128)], list(range(128)))
    out, lse = c.attn()
    c.check(out, lse, c.own, "every length")


@pytest.mark.parametrize("dtype", [BF, FS])
def test_the_largest_tables(dtype):
    """64 sequences, 64 KV heads, 64 shared caches: 4096 segments of either kind."""
    rng = np.random.default_rng(8)
    c = Case(dtype, 1, 64, 64, [63 - b for b in range(64)], [int(n) for n in rng.integers(0, 40, 4096)], [int(n) for n in rng.integers(0, 12, 4096)])
    out, lse = c.attn()
    c.check(out, lse, c.own, "4096 segments")


def test_nothing_shared_and_nothing_at_all():
    c = Case(BF, 4, 2, 128, [-1, 0, -1], [0, 0], [0, 5, 0, 0, 3, 0])
    out, lse = c.attn()
    c.check(out, lse, c.own, "empty segments")
    assert not out[0, :4].any() and not out[1].any() and torch.isneginf(lse[1]).all()
    c = Case(BF, 4, 2, 128, [-1, -1], [40, 50], [100, 5, 70, 3])
    out, lse = c.attn()
    c.check(out, lse, c.own, "no sequence shares")
    plain, plain_lse = adakv.decode_attn(c.layer, c.q, c.cu, c.headroom, c.K, c.V, c.lens, want_lse=True)
    c.check(plain, plain_lse, c.own, "decode_attn")


def test_lengths_that_cannot_be():
    """A length below 0 counts as 0, one beyond the capacity as the capacity, here as in the other steps."""
    c = Case(BF, 4, 2, 64, [0, 0, 0], [50, 90], [8] * 6)
    c.p_lens.copy_(torch.tensor([-5, 2 ** 31 - 1], dtype=torch.int32))
    c.shared = [0, 90]
    out, lse = c.attn()
    c.check(out, lse, c.own, "lengths")


@pytest.mark.parametrize("batch", [2, 8, 20, 40])
@pytest.mark.parametrize("dtype", [BF, FH, FS])
def test_large_and_small_logits(dtype, batch):
    """Weights far apart, in either order: the reference moves, and parts meet that differ by any factor."""
    c = Case(dtype, 4, 1, 64, [0] * batch, [700], [20] * batch, q_by=30.0)
    for flip in (False, True):
        order = torch.argsort(f64_norm(c.pK[:700]), descending=flip)
        c.pK[:700], c.pV[:700] = c.pK[order], c.pV[order]
        out, lse = c.attn()
        c.check(out, lse, c.own, f"flip {flip}")


def f64_norm(t):
    return t.double().norm(dim=1)


@pytest.mark.parametrize("batch", [2, 8, 20, 40])
@pytest.mark.parametrize("dtype", [BF, FH, FS])
def test_logits_of_two_to_the_26(dtype, batch):
    """2^26 less 0, 4, 8 or 12, all of them fp32 numbers, in shared and own segments and in the appended row."""
    c = Case(dtype, 4, 1, 64, [0] * batch, [200], [9] * batch)
    c.layer = adakv.Layer(dtype, 4, 1, 64, 1, 7, 0.2, [9] * batch, [9] * batch, scale=1.0)
    less = 4 * torch.randint(0, 4, (200 + 10 * batch,), generator=torch.Generator().manual_seed(5))
    seen = torch.zeros(len(less), 64)
    seen[:, 0], seen[:, 1] = 2.0 ** 13, -less.float()
    seen = seen.to(dtype).to(DEV)
    c.pK[:200], c.k[:, 0] = seen[:200], seen[200:200 + batch]
    c.q.zero_()
    c.q[..., 0], c.q[..., 1] = 2.0 ** 13, 1.0
    own = seen[200 + batch:].view(batch, 9, 64)
    starts = D.segment_starts(c.cu.cpu().numpy(), c.headroom)
    for b in range(batch):
        c.K[starts[b]:starts[b] + 9] = own[b]
    out, lse = c.step()
    for b in range(batch):
        w = torch.exp(-torch.cat([less[:200], less[200 + batch + 9 * b:][:9], less[200 + b:][:1]]).double())
        V = torch.cat([c.pV[:200], c.V[starts[b]:starts[b] + 9], c.v[b]]).double().cpu()
        want, mag = (w[:, None] * V).sum(0) / w.sum(), (w[:, None] * V.abs()).sum(0) / w.sum()
        # exponents of up to 2^26 log2 e, of which 17.4 are the largest difference and up to 9 a reference's rounding or its bias: off by 2^-20
        # at most, with the factor log2 e by 17.4 * 2^-25 more; a weight is cut to 2^-23, and 210 of them are added
        error = 2.0 ** -19 + 17.4 * 2.0 ** -25 + 2.0 ** -23 + 2 * 210 * 2.0 ** -24
        assert ((out[b].double().cpu() - want).abs() <= 2 * error * mag).all(), f"sequence {b}"
        assert ((lse[b].double().cpu() - 2.0 ** 26).abs() <= 16).all()


@pytest.mark.parametrize("batch", [2, 8, 12, 20])
@pytest.mark.parametrize("dtype,d", [(BF, 128), (FH, 64), (FH, 128), (FS, 64), (FS, 128)])
def test_values_that_are_no_numbers(dtype, d, batch):
    """An infinite value makes its column infinite, NaN (or infinities of both signs) NaN; other columns and heads stay."""
    c = Case(dtype, 4, 2, d, [0] * (batch - 1) + [-1], [333, 100], [20] * (2 * batch), seed=3)
    want, want_lse = c.attn()
    c.pV[7, 3], c.pV[300, 5], c.pV[332, 40], c.pV[9, 9], c.pV[200, 9] = math.inf, -math.inf, math.nan, math.inf, -math.inf
    c.pV[332, 17] = math.inf                                   # (the last row, which the rows past a tile's end repeat)
    out, lse = c.attn()
    first = torch.zeros_like(out, dtype=torch.bool)
    first[:batch - 1, :4] = True
    cols = torch.zeros(d, dtype=torch.bool, device=DEV)
    cols[[3, 5, 40, 9, 17]] = True
    hit = first & cols
    assert torch.equal(out[~hit], want[~hit]) and torch.equal(lse, want_lse)
    got = out[:batch - 1, :4]
    assert (got[..., 3] == math.inf).all() and (got[..., 5] == -math.inf).all() and (got[..., 17] == math.inf).all()
    assert got[..., 40].isnan().all() and got[..., 9].isnan().all()


@pytest.mark.parametrize("batch", [2, 8, 20])
@pytest.mark.parametrize("dtype", [BF, FH, FS])
def test_logits_that_are_no_numbers(dtype, batch):
    """NaN and +inf make the heads that see the row NaN; -inf has no weight, and NaN where there is nothing else."""
    c = Case(dtype, 4, 1, 64, [0] * (batch - 1) + [-1], [200], [1] * batch, seed=4)
    c.q.abs_()
    c.pK[50] = math.nan
    out, lse = c.attn()
    assert out[:-1].isnan().all() and lse[:-1].isnan().all() and out[-1].isfinite().all()
    c.pK[50] = math.inf
    out, lse = c.attn()
    assert out[:-1].isnan().all() and lse[:-1].isnan().all() and out[-1].isfinite().all()
    c.pK[50] = -math.inf
    out, lse = c.attn()
    keep = [i for i in range(200) if i != 50]
    kept = c.pK.clone(), c.pV.clone()
    c.pK[:199], c.pV[:199] = kept[0][keep], kept[1][keep]
    c.shared = [199]
    c.check(out, lse, c.own, "a row without weight")
    c.pK[:200] = -math.inf
    c.K[:] = -math.inf
    out, lse = c.attn()
    assert out.isnan().all() and torch.isneginf(lse).all()


def test_large_values_are_summed_without_overflow():
    """Values times rows just below 2^127 (and a reference that lies below the largest logit for a while)."""
    c = Case(BF, 4, 1, 64, [0] * 5, [512], [1] * 5)
    c.pV.copy_((c.pV > 0).to(BF) * 2.0 ** 117)
    c.pK.mul_(torch.linspace(0.1, 1.5, 512, device=DEV)[:, None].to(BF))
    out, lse = c.attn()
    c.check(out, lse, c.own, "large values")


@pytest.mark.parametrize("batch", [3, 40])
def test_shared_caches_beyond_four_gigabytes(batch):
    rows, d, h = 17_000_000, 128, 2
    kept = [rows, 300]
    layer = adakv.Layer(BF, 8, h, d, 1, 7, 0.2, [rows], [sum(kept)])
    K = torch.empty((sum(kept), d), dtype=BF, device=DEV)
    V = torch.empty((sum(kept), d), dtype=BF, device=DEV)
    gen = torch.Generator().manual_seed(9)
    c = Case(BF, 4, h, d, [0] * batch, [5, 5], [9] * (h * batch))
    for t in (K, V):
        t[:200] = torch.randn((200, d), generator=gen).to(BF).to(DEV)
        t[rows:] = torch.randn((300, d), generator=gen).to(BF).to(DEV)
    c.shared, c.shared_headroom = [200, 300], 0
    c.pK, c.pV, c.p_cu = K, V, torch.tensor([0, rows, rows + 300], dtype=torch.int32, device=DEV)
    c.prefix = adakv.Prefix(layer, c.p_cu, 0, K, V, torch.tensor([200, 300], dtype=torch.int32, device=DEV), c.of)
    out, lse = c.attn()
    c.check(out, lse, c.own, "beyond 4 GB")


@pytest.mark.parametrize("batch", [4, 24])
def test_captured_with_lengths_that_grow(batch):
    """Two graphs that share a workspace, replayed in turn with eager calls in between."""
    made = [Case(BF, 4, 2, 128, [0] * batch, [500, 300], [6] * (2 * batch), headroom=12, shared_headroom=50, seed=s) for s in (1, 2)]
    ws = torch.zeros(max(adakv.prefix_workspace_bytes(c.layer, c.headroom, c.prefix) for c in made), dtype=torch.uint8, device=DEV)
    overflow = torch.zeros(1, dtype=torch.int32, device=DEV)
    graphs = []
    for c in made:
        c.out, c.lse = torch.zeros(batch, 8, 128, device=DEV), torch.zeros(batch, 8, device=DEV)
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            c.step(overflow=overflow, out=c.out, lse=c.lse, ws=ws)
        graphs.append(g)
    for turn in range(4):
        for c, g in zip(made, graphs):
            c.k.mul_(1.1)
            K, V, lens = c.K.clone(), c.V.clone(), c.lens.clone()
            g.replay()
            want, want_lse = adakv.decode_prefix_step(c.layer, c.q, c.k, c.v, c.cu, c.headroom, K, V, lens, c.prefix, want_lse=True)
            torch.cuda.synchronize()
            assert torch.equal(c.out, want) and torch.equal(c.lse, want_lse) and torch.equal(c.lens, lens), turn
            assert torch.equal(c.K.view(torch.uint8), K.view(torch.uint8))
            # the shared caches grow too: a later part of the prompt joins them
            starts = D.segment_starts(c.p_cu.cpu().numpy(), 50)
            for s, a in enumerate(starts):
                n = c.shared[s]
                c.pK[a + n:a + n + 9], c.pV[a + n:a + n + 9] = c.pK[a:a + 9] * 1.5, c.pV[a:a + 9]
                c.shared[s] += 9
            c.p_lens.add_(9)
        for c in made:
            c.check(*c.attn(), c.lens.cpu().numpy(), f"turn {turn}")
    assert overflow.item() == 0


def test_on_another_stream():
    c = Case(BF, 4, 2, 128, [0] * 9, [500, 300], [6] * 18)
    want, want_lse = c.attn()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    out, lse = c.attn(stream=side)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(out, want) and torch.equal(lse, want_lse)


def test_two_streams_over_one_shared_cache():
    """Two batches at once, each with a cache and a workspace of its own, read the same shared one."""
    c = Case(BF, 4, 2, 128, [0] * 20, [5000, 3000], [40] * 40)
    made = [(c.K.clone(), c.V.clone(), c.lens.clone()) for _ in range(3)]
    step = lambda t, **kw: adakv.decode_prefix_step(c.layer, c.q, c.k, c.v, c.cu, c.headroom, *t, c.prefix, want_lse=True, **kw)
    want, want_lse = step(made[0])
    sides = [torch.cuda.Stream() for _ in range(2)]
    for side in sides:
        side.wait_stream(torch.cuda.current_stream())
    got = [step(t, stream=side) for t, side in zip(made[1:], sides)]
    torch.cuda.synchronize()
    for (out, lse), t in zip(got, made[1:]):
        assert torch.equal(out, want) and torch.equal(lse, want_lse)
        assert all(torch.equal(x.view(torch.uint8), y.view(torch.uint8)) for x, y in zip(t, made[0]))


def test_results_do_not_change_from_run_to_run():
    c = Case(BF, 8, 2, 128, [0] * 30, [3000, 900], [70] * 60)
    want, want_lse = c.attn()
    for _ in range(5):
        out, lse = c.attn()
        assert torch.equal(out, want) and torch.equal(lse, want_lse)


def test_both_checks_make_the_same_call(monkeypatch):
    from paper_2407_11550_amd import binding
    results = []
    for native in (True, False):
        c, calls = Case(FH, 4, 2, 64, [0, -1, 0], [90, 30], [6] * 6), []
        ws = torch.zeros(adakv.prefix_workspace_bytes(c.layer, c.headroom, c.prefix), dtype=torch.uint8, device=DEV)
        out, over = torch.zeros(3, 8, 64, device=DEV), torch.zeros(1, dtype=torch.int32, device=DEV)
        if native:
            fn = binding._native
            monkeypatch.setattr(binding, "_native", lambda *a, **kw: calls.append(fn(*a, **kw)) or calls[-1])
        else:
            monkeypatch.setattr(binding, "_marshal", None)
        c.step(overflow=over, out=out, ws=ws, want_lse=False)
        torch.cuda.synchronize()
        assert not native or calls == [True]
        monkeypatch.undo()
        results.append([out, c.K, c.V, c.lens, over])
    for x, y in zip(*results):
        assert torch.equal(x.view(torch.uint8), y.view(torch.uint8))


def test_spoiled_arguments_are_refused_as_in_python(monkeypatch):
    from paper_2407_11550_amd import binding
    c = Case(BF, 4, 2, 64, [0, -1, 0], [90, 30], [6] * 6)
    ws = torch.zeros(adakv.prefix_workspace_bytes(c.layer, c.headroom, c.prefix), dtype=torch.uint8, device=DEV)
    good = dict(q_new=c.q, k_new=c.k, v_new=c.v, cu_seqlens=c.cu, headroom=c.headroom, K_cache=c.K, V_cache=c.V, seg_len=c.lens, prefix=c.prefix,
                overflow=None, out=torch.zeros(3, 8, 64, device=DEV), lse=torch.zeros(3, 8, device=DEV), ws=ws)
    other = Case(BF, 4, 2, 64, [0, -1], [90, 30], [6] * 4).prefix
    typed = Case(FH, 4, 2, 64, [0, -1, 0], [90, 30], [6] * 6).prefix
    own = adakv.Prefix(c.layer, c.cu, c.headroom, c.K, c.V, c.lens, [0, -1, 0])
    for what, bad in (("q", dict(q_new=c.q.cpu())), ("k", dict(k_new=c.k.float())), ("v", dict(v_new=c.v[:2])), ("headroom", dict(headroom=4)),
                      ("negative", dict(headroom=-1)), ("rows", dict(K_cache=c.K[:-1])), ("type", dict(V_cache=c.V.half())), ("lens", dict(seg_len=c.lens.long())),
                      ("cu", dict(cu_seqlens=c.cu[:6])), ("batch", dict(prefix=other)), ("shared type", dict(prefix=typed)), ("own cache", dict(prefix=own)),
                      ("ws", dict(ws=ws[:-300])), ("ws type", dict(ws=ws.view(torch.int32))), ("out", dict(out=good["out"][:2])), ("lse", dict(lse=good["lse"].double()))):
        said = []
        for native in (True, False):
            with monkeypatch.context() as m:
                if not native:
                    m.setattr(binding, "_marshal", None)
                with pytest.raises((ValueError, adakv.AdaKVError)) as e:
                    adakv.decode_prefix_step(c.layer, **{**good, **bad})
                said.append(str(e.value))
        assert said[0] == said[1], what
    torch.cuda.synchronize()

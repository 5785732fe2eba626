"""Shared and own segments in parts of many tiles, against 64 bits: what has short segments in the other tests."""
import math

import numpy as np
import pytest
import torch

import paper_2407_11550_amd as adakv
from oracle import decode_oracle as D
from oracle import serve_oracle as S
from prefix_parts import own_parts, plan, shared_parts
from serve_util import DEV, attention_bound, f64, lse_bound
from test_gpu_prefix import BF, FH, FS, Case

pytestmark = pytest.mark.gpu
NAMES = {BF: "bf16", FH: "fp16", FS: "fp32"}


def model(c):
    return plan(NAMES[c.dtype], c.d, c.g, c.h, c.of, len(c.shared) // c.h, c.cu.diff().tolist(), c.headroom)


def check_some(c, out, lse, held, sequences, heads=None):
    """Case.check for some sequences and KV heads alone."""
    for b in sequences:
        for h in range(c.h) if heads is None else heads:
            s = b * c.h + h
            Ks, Vs = c.rows(s, int(held[s]))
            for i in range(c.g):
                at = h * c.g + i
                ref, z, mag, big = S.attend(f64(c.q[b, at]), Ks, Vs, 1 / math.sqrt(c.d))
                keys = np.array(len(Ks))
                bound = attention_bound(c.dtype, c.d, ref, mag, np.array(big), np.array(z), keys, rounded=False)
                bound = bound + (mag * 2.0 ** -23 if c.dtype != FS else 0.0) + (len(Ks) * 2.0 ** -45 * np.abs(Vs).max() if c.dtype == FH else 0.0)
                assert (np.abs(f64(out[b, at]) - ref) <= bound).all(), (b, h, i)
                assert abs(float(lse[b, at]) - z) <= lse_bound(c.d, np.array(big), np.array(z), keys), (b, h, i)


def own_case(dtype, d, batch, seed=0):
    """Two KV heads; a cache of some 80000 rows for the sequences' own segments, which are held up to three quarters."""
    rng = np.random.default_rng(batch)
    room = 40000 // batch
    ends = [n + e for n in (0, 64, 128, 192, 256, 384) for e in (-1, 0, 1) if n + e >= 0]
    lens = [int(rng.choice(ends)) if rng.random() < 0.3 else int(rng.integers(0, 3 * room // 4)) for _ in range(2 * batch)]
    lens[:2] = [3 * room // 4, 3 * room // 4 - 1]
    c = Case(dtype, 4, 2, d, [0] * batch, [200, 70], [0] * (2 * batch), headroom=room, seed=seed)
    gen = torch.Generator().manual_seed(seed + 50)
    for a, n in zip(D.segment_starts(c.cu.cpu().numpy(), room), lens):
        for t in (c.K, c.V):
            t[a:a + n] = torch.randn((n, d), generator=gen).to(dtype).to(DEV)
    c.own = lens
    c.lens.copy_(torch.tensor(lens, dtype=torch.int32))
    return c


@pytest.mark.parametrize("batch", [64, 40, 12, 4])      # shared query rows: two blocks of 128, blocks of 128 and of 64, and 16 or 32
@pytest.mark.parametrize("dtype,d", [(t, d) for t in (BF, FH, FS) for d in (64, 128)])
def test_own_parts_of_several_tiles(dtype, d, batch):
    """Attention and then a step, whose rows are appended in the middle of a tile or begin one."""
    c = own_case(dtype, d, batch)
    p = model(c)
    assert max(n for _, _, n in own_parts(p, c.own)) > p["own_tile"]         # (a second tile, that is)
    out, lse = c.attn()
    check_some(c, out, lse, c.own, [0, 1, batch // 2, batch - 1])
    out, lse = c.step()
    assert c.lens.tolist() == [n + 1 for n in c.own]
    check_some(c, out, lse, c.lens.tolist(), [0, 1, batch - 2])


@pytest.mark.parametrize("batch", [64, 12, 4])
@pytest.mark.parametrize("dtype,d", [(t, d) for t in (BF, FH, FS) for d in (64, 128)])
def test_values_that_are_no_numbers_in_later_tiles_of_own_parts(dtype, d, batch):
    c = own_case(dtype, d, batch, seed=1)
    want, want_lse = c.attn()
    at, n = D.segment_starts(c.cu.cpu().numpy(), c.headroom)[0], c.own[0]
    tile = model(c)["own_tile"]
    c.V[at + tile + 1, 3], c.V[at + n - 1, 5], c.V[at + tile + 2, 40] = math.inf, -math.inf, math.nan
    c.V[at + tile - 1, 9], c.V[at + tile + 40, 9] = math.inf, -math.inf
    out, lse = c.attn()
    hit = torch.zeros_like(out, dtype=torch.bool)
    hit[0, :4, [3, 5, 40, 9]] = True
    assert torch.equal(out[~hit], want[~hit]) and torch.equal(lse, want_lse)
    got = out[0, :4]
    assert (got[:, 3] == math.inf).all() and (got[:, 5] == -math.inf).all() and got[:, 40].isnan().all() and got[:, 9].isnan().all()


@pytest.mark.parametrize("dtype", [BF, FH, FS])
def test_the_largest_logits_in_the_last_tiles_of_own_parts(dtype):
    """Own rows in the order of their size: the reference moves in every tile."""
    c = own_case(dtype, 128, 64, seed=2)
    c.q.mul_(8)
    for a, n in zip(D.segment_starts(c.cu.cpu().numpy(), c.headroom), c.own):
        c.K[a:a + n] = c.K[a:a + n] * torch.linspace(0.1, 2.0, n, device=DEV)[:, None].to(dtype)
    out, lse = c.attn()
    check_some(c, out, lse, c.own, [0, 1, 30, 63])


SHARED = [
    # dtype d  g  h sequences caches rows a head, times that parts are made longer
    (BF, 128, 4, 8, 64, 1, 6000, 1),            # two blocks of rows
    (BF, 64, 8, 8, 64, 1, 8000, 1),             # four
    (BF, 128, 4, 8, 8, 3, 4000, 1),             # one of 64
    (FH, 128, 4, 8, 48, 1, 8000, 1),
    (FS, 128, 8, 8, 28, 1, 4000, 1),
    (FS, 64, 8, 8, 40, 1, 4000, 1),
    (FS, 128, 4, 8, 8, 1, 4000, 1),             # 16 rows
    (BF, 128, 8, 32, 64, 1, 2500, 2),
    (BF, 64, 8, 64, 40, 1, 1000, 2),
    (FS, 128, 4, 64, 40, 1, 1000, 2),
    (BF, 128, 8, 8, 64, 9, 900, 0),             # more than 64 segments, which nothing makes longer
    (FH, 64, 8, 8, 64, 9, 900, 0),
    (FS, 128, 8, 8, 24, 9, 900, 0),
]


@pytest.mark.parametrize("dtype,d,g,h,batch,groups,rows,turns", SHARED)
def test_shared_parts_that_are_made_longer(dtype, d, g, h, batch, groups, rows, turns):
    """Uneven heads: parts of many tiles, as many as one to a compute unit, in groups of 8 where there are several blocks of query rows."""
    rng = np.random.default_rng(0)
    share = np.exp(rng.standard_normal(groups * h))
    lens = [max(1, int(n)) for n in rows * groups * h * share / share.sum()]
    of = [int(p) for p in rng.integers(0, groups, batch)]
    c = Case(dtype, g, h, d, of, lens, [int(n) for n in rng.integers(0, 30, batch * h)], headroom=64)
    got, split, found = shared_parts(model(c), h, lens)
    assert got == turns and max(n for _, _, n, _, _ in filter(None, found)) > model(c)["tile"] * min(3, split - 1)
    out, lse = c.attn()
    heads = sorted({0, 1, h - 1, int(np.argmax(lens[:h])), int(np.argmin(lens[:h]))})[:6]
    check_some(c, out, lse, c.own, [0, batch // 2, batch - 1], heads)
    some = [b for b in range(batch) if of[b] == of[0]][-1]                      # (the last block of rows)
    check_some(c, out, lse, c.own, [some], heads)


@pytest.mark.parametrize("batch,chains", [(2, 4), (12, 2), (40, 2)])
@pytest.mark.parametrize("d", [64, 128])
def test_logits_are_sums_of_short_chains(d, batch, chains):
    """2^24, then d - 2 products of 1 + 2^-4, then -2^24, in 32 bits: a chain that begins with 2^24 is off by nearly 1, half a step, with every
    product.  There are d / chains in it, and 2 roundings join the chains; own segments have four chains everywhere."""
    for of, lens, most in ((0, ([1], [0] * batch), d / chains), (-1, ([1], [1] * batch), d / 4)):
        c = Case(FS, 4, 1, d, [of] * batch, *lens)
        c.layer = adakv.Layer(FS, 4, 1, d, 1, 7, 0.2, [1] * batch, [1] * batch, scale=1.0)
        row = torch.ones(d, device=DEV)
        row[0], row[-1] = 2.0 ** 12, -2.0 ** 12
        c.q[:] = 1 + 2.0 ** -4
        c.q[..., 0] = c.q[..., -1] = 2.0 ** 12
        (c.pK if of == 0 else c.K).copy_(row)
        out, lse = c.attn()
        print(f"  of {of}: off by {float((lse - (d - 2) * 1.0625).abs().max())}, at most {most + 2}", flush=True)
        assert ((lse.double() - (d - 2) * 1.0625).abs() <= most + 2).all()

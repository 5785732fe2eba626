"""The rotary calls refuse outputs that have memory of another tensor of the call, on the host and before anything is launched; all others go through."""
import ctypes
import random
import time

import pytest
import torch

import paper_2407_11550_amd as adakv
from paper_2407_11550_amd import binding

A, WORD, HEAD = 1 << 30, 16, 8          # an address that is never looked at; bytes of a word, words of a head (bf16, d = 64)


def layer(h_q, h_kv, lens=(1,), tok_off=None):
    return adakv.Layer(torch.bfloat16, h_q, h_kv, 64, 1, 7, 0.2, [n - 1 if n > 1 else 1 for n in lens], [h_kv for _ in lens], tok_off=tok_off)


def heads(at, tok, head):
    """At a word, strides in words."""
    return binding._CHeads(A + at * WORD, tok * 8, head * 8)


def call(lib, L, rows, q, k, qo, ko, positions=1 << 50, freq=3 << 50, weights=(5 << 50, 7 << 50), dims=64):
    """-2: past the checks of places, at that of the weights' alignment behind them, so that nothing is launched."""
    assert weights[0] % 16 == 0
    rotation = binding._CRotation(0, dims, 1.0, freq)
    by = [None if h is None else ctypes.byref(h) for h in (q, k, qo, ko)]
    got = lib.adakv_norm_rotary(ctypes.byref(L.c), ctypes.byref(rotation), rows, positions, *by[:2], weights[0] + 8, weights[1], 1e-6, *by[2:], None)
    assert got in (-1, -2), got
    return got


def words(h, rows, count):
    at, tok, head = (h.x - A) // WORD, h.stride_tok // 8, h.stride_head // 8
    return [at + r * tok + i * head + e for r in rows for i in range(count) for e in range(HEAD)]


def wrong(q, k, qo, ko, h_q, h_kv, rows, reach):
    for x, o, n in ((q, qo, h_q), (k, ko, h_kv)):
        tok, head = o.stride_tok // 8, o.stride_head // 8
        if tok < (n - 1) * head + HEAD and head < (reach - 1) * tok + HEAD:
            return True                 # places of the output itself, whether they meet or not
        if x.x == o.x and (x.stride_tok, x.stride_head) != (o.stride_tok, o.stride_head):
            return True
    taken = {name: set(words(h, rows, n)) for name, h, n in (("q", q, h_q), ("k", k, h_kv), ("qo", qo, h_q), ("ko", ko, h_kv))}
    pairs = [("qo", "k"), ("ko", "q"), ("qo", "ko")] + [("qo", "q")] * (q.x != qo.x) + [("ko", "k")] * (k.x != ko.x)
    return any(taken[a] & taken[b] for a, b in pairs)


def test_against_the_sets_of_words(lib):
    rng = random.Random(11)
    said = [0, 0]
    for turn in range(6000):
        h_kv, g, rows = rng.choice([1, 2, 3]), rng.choice([1, 2]), rng.choice([1, 2, 3, 5, 12])
        h_q = g * h_kv
        far = rng.choice([40, 200, 2000])
        q, k, qo, ko = (heads(rng.randrange(far), *rng.choice([(rng.randrange(8, 60), 8), (rng.randrange(8, 60), rng.randrange(8, 90)),
                                                               (8, rng.randrange(8, 200)), (48, 8), (48, 16)])) for _ in range(4))
        if rng.random() < 0.4:
            qo = q
        if rng.random() < 0.4:
            ko = k
        bad = wrong(q, k, qo, ko, h_q, h_kv, range(rows), rows)
        said[bad] += 1
        assert call(lib, layer(h_q, h_kv), rows, q, k, qo, ko) == (-1 if bad else -2), (turn, rows, h_q, h_kv, [(h.x, h.stride_tok, h.stride_head) for h in (q, k, qo, ko)])
    assert min(said) > 500


def test_against_the_sets_of_words_in_sequences(lib):
    """Without positions: rows between sequences are no places."""
    rng = random.Random(12)
    said = [0, 0]
    for turn in range(3000):
        lens, off = [rng.randrange(2, 5) for _ in range(rng.randrange(1, 4))], [rng.randrange(3)]
        for n in lens:
            off.append(off[-1] + n + rng.choice([0, 0, 3, 6]))
        L = layer(2, 1, lens, off)
        rows = [r for a, n in zip(off, lens) for r in range(a, a + n)]
        reach = rows[-1] + 1
        at = rng.randrange(400)
        q = heads(at, 24, 8)
        qo = heads(at + 24 * rng.randrange(-8, 9) if rng.random() < 0.8 else 5000, 24, 8) if at >= 200 else q
        k = heads(at + 16 if rng.random() < 0.5 else 2000 + rng.randrange(300), 24, 8)
        ko = k if rng.random() < 0.5 else heads(rng.randrange(3000), rng.choice([24, 8, 11]), 8)
        bad = wrong(q, k, qo, ko, 2, 1, rows, reach)
        said[bad] += 1
        assert call(lib, L, 0, q, k, qo, ko, positions=None) == (-1 if bad else -2), turn
    assert min(said) > 300


def test_parts_of_one_tensor(lib):
    """In place within fused rows, and the places that are none's; 2^29 rows, for which nothing is gone through one by one."""
    L, rows = layer(32, 8), 1 << 29
    tok = 48 * HEAD
    q, k, v = (heads(i * HEAD, tok, HEAD) for i in (0, 32, 40))
    assert call(lib, L, rows, q, k, q, k) == -2
    assert call(lib, L, rows, q, k, q, v) == -2
    assert call(lib, L, rows, q, k, k, v) == -1              # queries' heads are more than the keys'
    assert call(lib, L, rows, q, k, q, heads(39 * HEAD, tok, HEAD)) == -1
    assert call(lib, L, rows, q, k, heads(tok, tok, HEAD), k) == -1          # a row further on
    assert call(lib, L, rows, q, k, heads(tok * rows, tok, HEAD), k) == -2
    assert call(lib, L, rows, q, k, heads(tok * (rows - 1), tok, HEAD), k) == -1
    assert call(lib, L, rows, q, k, q, heads(32 * HEAD + 1, tok, HEAD)) == -1
    # rows of other distances that pass each other by, and that do not
    wide = heads(40 * HEAD, 3 * tok, HEAD)
    assert call(lib, L, rows, q, k, q, wide) == -2
    assert call(lib, L, rows, q, k, q, heads(40 * HEAD, tok + HEAD, HEAD)) == -1
    # one head in 8 of a cache with heads outermost
    outer = heads(1 << 20, HEAD, HEAD * 4096)
    assert call(lib, L, 4096, q, k, q, outer) == (-1 if (1 << 20) < tok * 4096 else -2)


def test_vectors_among_the_outputs(lib):
    L, rows = layer(4, 2), 10
    q, k, qo, ko = (heads(i * 4000, (4, 2)[i % 2] * HEAD, HEAD) for i in range(4))
    last = A + (8000 + 10 * 32) * WORD                       # behind q_out
    assert call(lib, L, rows, q, k, qo, ko) == -2
    for at, size in ((last - 16, 1), (qo.x, 1), (ko.x + 640, 1), (ko.x - 16, 1)):
        assert call(lib, L, rows, q, k, qo, ko, positions=at) == -1
        assert call(lib, L, rows, q, k, qo, ko, freq=at) == -1
        assert call(lib, L, rows, q, k, qo, ko, freq=at, dims=0) == -2       # not read
        assert call(lib, L, rows, q, k, qo, ko, weights=(at, 7 << 50)) == -1
        assert call(lib, L, rows, q, k, qo, ko, weights=(5 << 50, at)) == -1
    assert call(lib, L, rows, q, k, qo, ko, positions=last, freq=qo.x - 256, weights=(ko.x - 144, last + 64)) == -2
    assert call(lib, L, rows, q, None, qo, None, weights=(5 << 50, qo.x)) == -2           # not read either


def test_many_heads_of_other_distances(lib):
    """What cannot be told within a moment is refused before it is looked for."""
    L = adakv.Layer(torch.bfloat16, 4096, 1, 64, 1, 7, 0.2, [1], [1])
    begin = time.perf_counter()
    for rows, said in ((5, -1), (5000, -2)):                 # (a few rows can be told)
        assert call(lib, L, rows, heads(0, 1 << 20, 24), heads(1 << 40, 8, 8), heads(8, 1 << 21, 40), heads(1 << 41, 8, 8)) == said
    assert time.perf_counter() - begin < 1


@pytest.mark.gpu
def test_from_python():
    L, rot = layer(4, 2), adakv.Rotary(64)
    x = torch.zeros(30, 6, 64, dtype=torch.bfloat16, device="cuda:0")
    q, k, pos = x[:20, :4], x[:20, 4:], torch.arange(20, dtype=torch.int32, device="cuda:0")
    for bad in (dict(q_out=x[1:21, :4], k_out=k), dict(q_out=q, k_out=x[10:30, 4:]), dict(q_out=x[:20, 2:], k_out=k), dict(q_out=q, k_out=x[:20, :2])):
        with pytest.raises(adakv.AdaKVError) as e:
            adakv.rotary(L, rot, q, k, positions=pos, **bad)
        assert e.value.status == -1
    adakv.rotary(L, rot, q[:10], k[:10], positions=pos[:10], q_out=x[10:20, :4], k_out=x[20:, 4:])
    torch.cuda.synchronize()

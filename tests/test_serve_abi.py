"""What the calls around a served cache refuse, on the host and before anything is launched; and what their oracle is."""
import ctypes

import numpy as np
import pytest
import torch

import paper_2407_11550_amd as adakv
from oracle import decode_oracle as D
from oracle import serve_oracle as S

ONE = ctypes.c_void_p(1 << 20)      # never dereferenced: validation comes first
ODD = ctypes.c_void_p((1 << 20) + 8)
BIG = 1 << 30


def layer(**kw):
    args = dict(dtype=torch.bfloat16, h_q=32, h_kv=8, d=128, w=32, pool_k=7, alpha=0.2, n=[4096], B=[8 * 160])
    args.update(kw)
    return adakv.Layer(**args)


def test_the_calls_are_there(lib):
    for name in ("window_attn", "decode_window_attn", "decode_window_step", "q8_scales", "cache_build_q8", "append_q8",
                 "decode_attn_q8", "decode_step_q8", "cache_move", "cache_move_q8"):
        assert hasattr(lib, "adakv_" + name), name


def test_window_attn_refusals(lib):
    def call(L=layer(), q=ONE, tok=4096, head=128, K=ONE, V=ONE, window=16, sinks=1, out=ONE):
        return lib.adakv_window_attn(ctypes.byref(L.c), q, tok, head, K, V, window, sinks, out, None, None)

    for bad in (dict(window=0), dict(window=-3), dict(sinks=-1), dict(tok=127), dict(head=64), dict(q=None), dict(K=None), dict(V=None),
                dict(out=None), dict(L=layer(w=0)), dict(L=layer(h_q=30))):
        assert call(**bad) == -1, bad
    for bad in (dict(q=ODD), dict(K=ODD), dict(V=ODD), dict(out=ODD), dict(tok=4100), dict(head=132), dict(L=layer(d=96)), dict(L=layer(k_strides=(1 << 23, 128))), dict(L=layer(v_strides=(1 << 23, 128))),
                dict(L=layer(n=[(1 << 28) - 31], h_q=1, h_kv=1, B=[64])), dict(L=layer(n=[(1 << 27)] * 2, h_q=32, h_kv=1, B=[64] * 2))):
        assert call(**bad) == -2, bad


def test_decode_window_refusals(lib):
    L, by = layer(), ctypes.byref(layer().c)
    attn, step = lib.adakv_decode_window_attn, lib.adakv_decode_window_step
    assert attn(by, ONE, ONE, 4, ONE, ONE, ONE, 0, 0, ONE, None, ONE, BIG, None) == -1
    assert attn(by, ONE, ONE, 4, ONE, ONE, ONE, 5, -1, ONE, None, ONE, BIG, None) == -1
    assert attn(by, ONE, ONE, -1, ONE, ONE, ONE, 5, 0, ONE, None, ONE, BIG, None) == -1
    assert attn(by, ONE, ONE, 4, ONE, ONE, None, 5, 0, ONE, None, ONE, BIG, None) == -1
    assert attn(by, ONE, ONE, 4, ONE, ODD, ONE, 5, 0, ONE, None, ONE, BIG, None) == -2
    need = adakv.decode_workspace_bytes(L, 4)
    assert attn(by, ONE, ONE, 4, ONE, ONE, ONE, 5, 0, ONE, None, ONE, need - 1, None) == -3
    assert step(by, ONE, None, ONE, ONE, 4, ONE, ONE, ONE, None, 5, 0, ONE, None, ONE, BIG, None) == -1
    assert step(by, ONE, ONE, ONE, ONE, 4, ONE, ONE, ONE, None, 0, 0, ONE, None, ONE, BIG, None) == -1
    assert step(by, ONE, ODD, ONE, ONE, 4, ONE, ONE, ONE, None, 5, 0, ONE, None, ONE, BIG, None) == -2
    assert attn(ctypes.byref(layer(h_q=24).c), ONE, ONE, 4, ONE, ONE, ONE, 5, 0, ONE, None, ONE, BIG, None) == -2


def test_q8_refusals(lib):
    L, by = layer(), ctypes.byref(layer().c)
    rows = adakv.cache_rows(L, 5)
    assert adakv.q8_scales(L, 5) == rows // 32 + 8
    assert lib.adakv_q8_scales(by, -1) == 0 and lib.adakv_q8_scales(ctypes.byref(layer(w=0).c), 5) == 0
    good = [by, ONE, ONE, ONE, ONE, 4, ONE, ONE, ONE, ONE, ONE, None]
    for at in (1, 2, 3, 4, 6, 7, 8, 9, 10):
        assert lib.adakv_cache_build_q8(*[None if i == at else a for i, a in enumerate(good)]) == -1, at
    for at in (1, 2, 6, 7):
        assert lib.adakv_cache_build_q8(*[ODD if i == at else a for i, a in enumerate(good)]) == -2, at
    assert lib.adakv_cache_build_q8(*[-1 if i == 5 else a for i, a in enumerate(good)]) == -1
    assert lib.adakv_cache_build_q8(*[1 << 30 if i == 5 else a for i, a in enumerate(good)]) == -2
    good = [by, ONE, ONE, ONE, 4, ONE, ONE, ONE, ONE, ONE, None, None]
    for at in (1, 2, 3, 5, 6, 7, 8, 9):
        assert lib.adakv_append_q8(*[None if i == at else a for i, a in enumerate(good)]) == -1, at
    good = [by, ONE, ONE, 4, ONE, ONE, ONE, ONE, ONE, ONE, None, ONE, BIG, None]
    for at in (1, 2, 4, 5, 6, 7, 8, 9):
        assert lib.adakv_decode_attn_q8(*[None if i == at else a for i, a in enumerate(good)]) == -1, at
    need = adakv.decode_workspace_bytes(L, 4)
    assert lib.adakv_decode_attn_q8(*good[:12], need - 1, None) == -3
    assert lib.adakv_decode_attn_q8(*good[:11], None, BIG, None) == -3
    good = [by, ONE, ONE, ONE, ONE, 4, ONE, ONE, ONE, ONE, ONE, None, ONE, None, ONE, BIG, None]
    for at in (1, 2, 3, 4, 6, 7, 8, 9, 10, 12):
        assert lib.adakv_decode_step_q8(*[None if i == at else a for i, a in enumerate(good)]) == -1, at
    for at in (1, 2, 3, 6, 7):
        assert lib.adakv_decode_step_q8(*[ODD if i == at else a for i, a in enumerate(good)]) == -2, at
    assert lib.adakv_decode_step_q8(ctypes.byref(layer(h_q=24).c), *good[1:]) == -2


def test_cache_move_refusals(lib):
    L = layer(n=[100, 100], B=[8 * 40, 8 * 50])
    by = ctypes.byref(L.c)
    at = lambda i: ctypes.c_void_p((1 << 24) * (i + 1))          # far apart
    i32 = lambda *v: (ctypes.c_int32 * len(v))(*v)
    good = [by, 2, i32(1, 0), at(0), 4, at(1), at(2), at(3), 9, at(4), at(5), at(6), at(7), None, None]
    for k in (2, 3, 5, 6, 7, 9, 10, 11, 12):
        assert lib.adakv_cache_move(*[None if i == k else a for i, a in enumerate(good)]) == -1, k
    for k, v in ((1, 0), (1, 65), (2, i32(2, 0)), (2, i32(0, -1)), (4, -1), (8, -1)):
        assert lib.adakv_cache_move(*[v if i == k else a for i, a in enumerate(good)]) == -1, (k, v)
    assert lib.adakv_cache_move(*[1 << 28 if i == 8 else a for i, a in enumerate(good)]) == -2
    for k in (5, 6, 10, 11):
        assert lib.adakv_cache_move(*[ctypes.c_void_p((1 << 27) + 8) if i == k else a for i, a in enumerate(good)]) == -2, k
    # the last byte of one buffer and the first of another
    rows, out = adakv.cache_rows(L, 4) * 256, adakv.cache_rows(L.pick([1, 0]), 9) * 256
    over = lambda k, v: lib.adakv_cache_move(*[ctypes.c_void_p(v) if i == k else a for i, a in enumerate(good)])
    assert over(10, at(1).value + rows - 16) == -1 and over(10, at(2).value - out + 16) == -1 and over(11, at(5).value) == -1
    assert over(9, at(0).value + 64) == -1 and over(12, at(3).value) == -1 and over(12, at(5).value + 128) == -1
    good8 = [by, 1, i32(1), at(0), 4, at(1), at(2), at(3), at(4), at(5), 9, at(6), at(7), at(8), at(9), at(10), at(11), None, None]
    for k in (7, 8, 14, 15):
        assert lib.adakv_cache_move_q8(*[None if i == k else a for i, a in enumerate(good8)]) == -1, k
    assert lib.adakv_cache_move_q8(*[at(4) if i == 14 else a for i, a in enumerate(good8)]) == -1


def test_the_binding_refuses_what_the_kernels_would_miss(lib):
    L = layer(n=[100], B=[8 * 40])
    bf, f8 = torch.bfloat16, torch.float8_e4m3fn
    K, q = torch.zeros(132, 8, 128, dtype=bf), torch.zeros(132, 32, 128, dtype=bf)
    i32 = lambda k: torch.zeros(k, dtype=torch.int32)
    with pytest.raises(ValueError, match="window must be given"):
        adakv.window_attn(L, q, K, K, None)
    with pytest.raises(ValueError, match="window must be 1 or more"):
        adakv.window_attn(L, q, K, K, 0)
    with pytest.raises(ValueError, match="q must be"):
        adakv.window_attn(L, q[:, :31], K, K, 5)
    with pytest.raises(ValueError, match="contiguous rows"):
        adakv.window_attn(L, torch.zeros(132, 32, 256, dtype=bf)[:, :, ::2], K, K, 5)
    with pytest.raises(ValueError, match="q has 131 tokens"):
        adakv.window_attn(L, q[:131], K, K, 5)
    with pytest.raises(ValueError, match="V reaches"):
        adakv.window_attn(L, q, K, K[:131], 5)
    with pytest.raises(ValueError, match="out holds"):
        adakv.window_attn(L, q, K, K, 5, out=torch.zeros(131, 32, 128, dtype=bf))
    with pytest.raises(ValueError, match="row_lse holds"):
        adakv.window_attn(L, q, K, K, 5, row_lse=torch.zeros(32 * 31))
    with pytest.raises(ValueError, match="device tensor"):
        adakv.window_attn(L, q, K, K, 5)
    flat, qn, kn = torch.zeros(320, 128, dtype=bf), torch.zeros(1, 32, 128, dtype=bf), torch.zeros(1, 8, 128, dtype=bf)
    with pytest.raises(ValueError, match="sinks need a window"):
        adakv.decode_attn(L, qn, i32(9), 0, flat, flat, i32(8), sinks=3, ws=torch.zeros(1 << 20, dtype=torch.uint8))
    with pytest.raises(ValueError, match="window must be 1 or more"):
        adakv.decode_step(L, qn, kn, kn, i32(9), 0, flat, flat, i32(8), window=-1, ws=torch.zeros(1 << 20, dtype=torch.uint8))
    cache = adakv.q8_cache(L, 3, "cpu")
    assert cache.K.shape == (344, 128) and cache.K.dtype == f8 and cache.k_scale.numel() == 344 // 32 + 8
    ws = torch.zeros(1 << 20, dtype=torch.uint8)
    with pytest.raises(ValueError, match="contiguous .rows, 128"):
        adakv.decode_attn_q8(L, qn, i32(9), 4, cache, i32(8), ws=ws)
    with pytest.raises(ValueError, match="k_scale holds"):
        adakv.decode_attn_q8(L, qn, i32(9), 3, cache._replace(k_scale=cache.k_scale[1:]), i32(8), ws=ws)
    with pytest.raises(ValueError, match="seg_len"):
        adakv.append_q8(L, kn, kn, i32(9), 3, cache, i32(7))
    with pytest.raises(ValueError, match="k_new and v_new"):
        adakv.append_q8(L, kn, kn[:, :7], i32(9), 3, cache, i32(8))
    with pytest.raises(ValueError, match="k_new and v_new"):
        adakv.decode_step_q8(L, qn, kn.transpose(1, 2), kn, i32(9), 3, cache, i32(8), ws=ws)
    with pytest.raises(ValueError, match="indices"):
        adakv.cache_build_q8(L, K, K, i32(319), i32(9), 3, cache, i32(8))
    with pytest.raises(ValueError, match="device tensor"):
        adakv.cache_build_q8(L, K, K, i32(320), i32(9), 3, cache, i32(8))
    with pytest.raises(ValueError, match="not valid"):
        adakv.q8_cache(L, -1, "cpu")
    for picks in ([], [1], [-1]):
        with pytest.raises(ValueError, match="picks"):
            adakv.cache_move(L, picks, i32(9), 0, flat, flat, i32(8), 0)
    with pytest.raises(ValueError, match="K_cache|contiguous"):
        adakv.cache_move(L, [0, 0], i32(9), 0, flat, flat, i32(8), 0, K_out=flat, V_out=flat)
    with pytest.raises(ValueError, match="len_out"):
        adakv.cache_move(L, [0], i32(9), 0, flat, flat, i32(8), 0, len_out=i32(7))


def test_tensors_of_another_device_are_refused(monkeypatch, lib):
    """(a stand-in for tensors on two devices)"""
    import types
    from paper_2407_11550_amd import binding
    on = lambda d: types.SimpleNamespace(is_cuda=True, get_device=lambda: d)
    monkeypatch.setattr(binding, "_current_device", lambda: 0)
    binding._one_device(None, a=on(0), b=None)
    with pytest.raises(ValueError, match="b is on device 1"):
        binding._one_device(None, a=on(0), b=on(1))
    stream = types.SimpleNamespace(device=torch.device("cuda", 1))
    binding._one_device(stream, b=on(1))
    with pytest.raises(ValueError, match="launched on 1"):
        binding._one_device(stream, a=on(0))


def test_the_picked_layer():
    L = layer(n=[100, 200], B=[8 * 40, 8 * 50], scale=0.3, v_strides=(4096, 256))
    P = L.pick([1, 0, 1])
    assert P.n == [200, 100, 200] and P.B == [400, 320, 400] and P.scale == L.scale and P.v_strides == L.v_strides
    assert P.strides_given == (False, True) and P.tok_off == [0, 232, 364, 596]


# ---- the oracle against things that are not it -----------------------------------------------------------
def test_oracle_rounding_is_that_of_the_format():
    x = torch.cat([torch.randn(5000) * 100, torch.randn(5000) * 0.01, torch.arange(-480, 480, 0.25)])
    want = x.clamp(-448, 448).to(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(S.round_e4m3(x.double().numpy()), want)
    assert np.isnan(S.round_e4m3([np.nan, np.inf, -np.inf])).all()


def test_oracle_exponents():
    assert [S.exponent(m) for m in (0.0, 448.0, np.nextafter(448, 500), 1.0, 1.75, 2.0 ** -61 * 448, 2.0 ** 120)] == [-60, 0, 1, -8, -8, -60, 100]


def test_oracle_windows_by_brute_force_and_as_library_attention():
    n, d = 23, 8
    q, K, V = (torch.randn(n, d, dtype=torch.float64, generator=torch.Generator().manual_seed(i)) for i in range(3))
    for window, sinks in ((1, 0), (5, 2), (40, 0), (3, 30)):
        seen = torch.tensor([[j <= i and (i - j < window or j < sinks) for j in range(n)] for i in range(n)])
        want = torch.nn.functional.scaled_dot_product_attention(q[None], K[None], V[None], attn_mask=seen)[0]
        out = S.prompt(q.numpy(), K.numpy(), V.numpy(), window, sinks, d ** -0.5)[0]
        assert np.allclose(out, want.numpy(), rtol=1e-12, atol=1e-14)
        for length in (0, 1, 6, 23):
            assert S.step_rows(length, window, sinks).tolist() == [j for j in range(length) if seen[length - 1][j]]


def test_oracle_append_is_a_build_where_scales_do_not_shrink():
    """Rows appended one by one are the built cache up to values that the growing scale rounded twice."""
    rng = np.random.RandomState(4)
    x = rng.randn(70, 8) * np.exp2(rng.randint(-3, 4, (70, 1)))
    codes, ks = S.quantise(x[:1])
    for row in x[1:]:
        codes, ks = S.append(codes, ks, row)
    built, kb = S.quantise(x)
    assert ks == kb
    step = np.exp2(np.maximum(np.floor(np.log2(np.abs(built) + 1e-30)) - 3, -9))
    assert (np.abs(built - codes) <= step).all() and (built != codes).mean() < 0.05
    assert np.abs(S.values(codes, ks) - x).max() <= 2.0 ** -4 * np.abs(x).max()


def test_oracle_move_by_hand():
    cu_out, lens, runs, over = S.move([1, 1], 1, [0, 4, 10], 2, [5, 8], 1)
    assert cu_out.tolist() == [0, 6, 12] and lens.tolist() == [7, 7] and over
    assert runs == [(6, 0, 7), (6, 7, 7)] and D.segment_starts([0, 4, 10], 2).tolist() == [0, 6]

"""What the calls over shared caches refuse, on the host and before anything is launched."""
import ctypes

import pytest
import torch

import paper_2407_11550_amd as adakv
from paper_2407_11550_amd import binding

A, BIG = 1 << 20, 1 << 34           # addresses that are never looked at: the checks come first
ODD = A + 8


def layer(**kw):
    args = dict(dtype=torch.bfloat16, h_q=32, h_kv=8, d=128, w=1, pool_k=7, alpha=0.2, n=[4096, 100], B=[8 * 160, 8])
    args.update(kw)
    return adakv.Layer(**args)


def shared(L=None, of=(0, 0), cu=A, headroom=0, K=BIG, V=2 * BIG, seg_len=3 * BIG):
    L = L or layer(n=[4096], B=[8 * 300])
    c = binding._CPrefix(ctypes.pointer(L.c), (ctypes.c_int32 * len(of))(*of), cu, headroom, K, V, seg_len)
    c.keep = L
    return c


def attn(lib, L=None, q=A, cu=A, headroom=4, K=A, V=A, lens=A, P=None, out=A, ws=A, ws_bytes=1 << 40):
    P = P if P is not None else shared()
    return lib.adakv_decode_prefix_attn(ctypes.byref((L or layer()).c), q, cu, headroom, K, V, lens, ctypes.byref(P), out, None, ws, ws_bytes, None)


def step(lib, L=None, q=A, k=A, v=A, cu=A, headroom=4, K=A, V=A, lens=A, P=None, out=A, ws=A, ws_bytes=1 << 40):
    P = P if P is not None else shared()
    return lib.adakv_decode_prefix_step(ctypes.byref((L or layer()).c), q, k, v, cu, headroom, K, V, lens, None, ctypes.byref(P), out, None, ws,
                                        ws_bytes, None)


@pytest.mark.parametrize("call", [attn, step])
def test_refusals(lib, call):
    assert call(lib, ws_bytes=0) == -3                     # all but the workspace as it has to be
    for bad in (dict(q=None), dict(cu=None), dict(K=None), dict(V=None), dict(lens=None), dict(out=None), dict(headroom=-1), dict(L=layer(w=0)),
                dict(L=layer(h_q=30)), dict(P=shared(of=(0, 1))), dict(P=shared(of=(-2, 0))), dict(P=shared(cu=None)), dict(P=shared(K=None)),
                dict(P=shared(V=None)), dict(P=shared(seg_len=None)), dict(P=shared(headroom=-1)), dict(P=shared(L=layer(w=0))),
                dict(P=shared(L=layer(dtype=torch.float16))), dict(P=shared(L=layer(h_q=16))), dict(P=shared(L=layer(h_kv=4, B=[1000, 4]))),
                dict(P=shared(L=layer(d=64)))):
        assert call(lib, **bad) == -1, bad
    for bad in (dict(q=ODD), dict(K=ODD), dict(V=ODD), dict(P=shared(K=ODD)), dict(P=shared(V=ODD)), dict(headroom=1 << 30),
                dict(P=shared(headroom=1 << 30)), dict(L=layer(h_q=24), P=shared(L=layer(h_q=24))), dict(L=layer(d=96), P=shared(L=layer(d=96)))):
        assert call(lib, **bad) == -2, bad
    need = adakv.load_library().adakv_prefix_workspace_bytes(ctypes.byref(layer().c), 4, ctypes.byref(shared()))
    assert need > 0
    assert call(lib, ws_bytes=need - 1) == -3 and call(lib, ws=None) == -3
    null = ctypes.POINTER(binding._CPrefix)()
    assert lib.adakv_decode_prefix_attn(ctypes.byref(layer().c), A, A, 4, A, A, A, null, A, None, A, BIG, None) == -1
    empty = shared()
    empty.L = ctypes.POINTER(binding._CLayer)()
    assert call(lib, P=empty) == -1
    empty = shared()
    empty.of = ctypes.POINTER(ctypes.c_int32)()
    assert call(lib, P=empty) == -1


def test_a_step_writes_into_no_shared_cache(lib):
    own = (8 * 160 + 8 + 16 * 4) * 256                     # bytes of the layer's own K_cache
    theirs = 8 * 300 * 256
    for K, V in ((A, 2 * BIG), (BIG, A), (A + own - 16, BIG), (BIG, A - theirs + 16)):
        assert step(lib, P=shared(K=K, V=V), V=4 * BIG, ws_bytes=0) == -1
        assert step(lib, P=shared(K=K, V=V), K=4 * BIG, ws_bytes=0) == -1
        assert attn(lib, P=shared(K=K, V=V), ws_bytes=0) == -3           # (reading is free)
    assert step(lib, P=shared(K=A + own, V=BIG), V=4 * BIG, ws_bytes=0) == -3
    for at in (A, A + 60, A - 28):                         # 16 lengths of its own, 8 of theirs
        assert step(lib, P=shared(seg_len=at), ws_bytes=0) == -1
        assert attn(lib, P=shared(seg_len=at), ws_bytes=0) == -3
    assert step(lib, P=shared(seg_len=A + 64), ws_bytes=0) == -3 and step(lib, P=shared(seg_len=A - 32), ws_bytes=0) == -3
    assert step(lib, k=None) == -1 and step(lib, v=None) == -1
    assert step(lib, k=ODD) == -2 and step(lib, v=ODD) == -2


def test_workspace_bytes(lib):
    def need(L=None, headroom=4, P=None):
        return lib.adakv_prefix_workspace_bytes(ctypes.byref((L or layer()).c), headroom, ctypes.byref(P or shared()))

    assert need(P=shared(of=(-1, -1))) > 0
    for bad in (dict(headroom=-1), dict(L=layer(w=0)), dict(P=shared(of=(0, 1))), dict(P=shared(headroom=-1)), dict(P=shared(L=layer(d=64))),
                dict(L=layer(h_q=24), P=shared(L=layer(h_q=24)))):
        assert need(**bad) == 0, bad
    # the largest batch and the largest shared caches: what a plan counts stays within its types
    many = layer(h_q=512, h_kv=64, n=[4096] * 64, B=[64] * 64)
    big = layer(h_q=512, h_kv=64, n=[500000] * 64, B=[31000000] * 64)
    assert 0 < need(many, P=shared(L=big, of=[i % 64 for i in range(64)])) < 1 << 36
    assert 0 < need(many, P=shared(L=big, of=[0] * 64)) < 1 << 36


def test_python_refusals(lib):
    L, S = layer(), layer(n=[4096], B=[8 * 300])
    K, cu, lens = torch.zeros(2400, 128, dtype=torch.bfloat16), torch.zeros(9, dtype=torch.int32), torch.zeros(8, dtype=torch.int32)
    for what, a in (("name the shared caches", dict(of=[0, 1])), ("name the shared caches", dict(of=[-2, 0])), ("K_cache", dict(K=K[:2399])),
                    ("V_cache", dict(V=K.view(1200, 256))), ("cu_seqlens", dict(cu=cu[:8])), ("seg_len", dict(lens=lens[:7])),
                    ("device tensor", dict())):
        kw = dict(dict(cu=cu, K=K, V=K, lens=lens, of=[0, 0]), **a)
        with pytest.raises(ValueError, match=what):
            adakv.Prefix(S, kw["cu"], 0, kw["K"], kw["V"], kw["lens"], kw["of"])
    assert L.batch == 2

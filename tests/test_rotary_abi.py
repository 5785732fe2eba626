"""What the rotary calls refuse, on the host and before anything is launched; and their frequencies."""
import ctypes
import math

import numpy as np
import pytest
import torch

import paper_2407_11550_amd as adakv
from oracle import rotary_oracle as R
from paper_2407_11550_amd import binding

A = 1 << 20                         # an address that is never looked at: the checks come first
ODD = A + 8


def layer(**kw):
    args = dict(dtype=torch.bfloat16, h_q=32, h_kv=8, d=128, w=32, pool_k=7, alpha=0.2, n=[4096], B=[8 * 160])
    args.update(kw)
    return adakv.Layer(**args)


def heads(x=A, tok=4096, head=128):
    return binding._CHeads(x, tok, head)


def rotation(layout=0, dims=128, magnitude=1.0, freq=A):
    return binding._CRotation(layout, dims, magnitude, freq)


def call(lib, norm=False, L=None, R=None, rows=0, positions=A, q="h", k="h", qo="h", ko="h", qw=A, kw=A, eps=1e-6):
    L, R = L or layer(), R or rotation()
    q, k, qo, ko = (heads(tok=1024 if i % 2 else 4096) if h == "h" else h for i, h in enumerate((q, k, qo, ko)))
    q, k, qo, ko = (None if h is None else ctypes.byref(h) for h in (q, k, qo, ko))
    if norm:
        return lib.adakv_norm_rotary(ctypes.byref(L.c), ctypes.byref(R), rows, positions, q, k, qw, kw, eps, qo, ko, None)
    return lib.adakv_rotary(ctypes.byref(L.c), ctypes.byref(R), rows, positions, q, k, qo, ko, None)


@pytest.mark.parametrize("norm", [False, True])
def test_refusals(lib, norm):
    assert call(lib, norm) == 0                            # no rows: nothing to do
    assert call(lib, norm, q=None, qo=None) == 0
    assert call(lib, norm, k=None, ko=None) == 0
    assert call(lib, norm, R=rotation(dims=0, freq=None)) == 0
    for bad in (dict(q=None), dict(ko=None), dict(q=None, qo=None, k=None, ko=None), dict(q=heads(None)), dict(ko=heads(None)),
                dict(rows=-1), dict(L=layer(w=0)), dict(L=layer(h_q=30)), dict(R=rotation(layout=2)), dict(R=rotation(dims=127)),
                dict(R=rotation(dims=130)), dict(R=rotation(dims=-2)), dict(R=rotation(freq=None)), dict(R=rotation(magnitude=-1.0)),
                dict(R=rotation(magnitude=math.inf)), dict(R=rotation(magnitude=math.nan)), dict(q=heads(tok=64)), dict(k=heads(head=64)),
                dict(qo=heads(head=-128)), dict(ko=heads(head=1 << 41)),
                dict(q=heads(), qo=heads(tok=8192)),                       # the same memory, other places
                dict(rows=3, qo=heads(A * 2, 128, 256)), dict(rows=3, ko=heads(A * 2, 512, 128))):   # places that meet
        assert call(lib, norm, **bad) == -1, bad
    for bad in (dict(q=heads(ODD)), dict(ko=heads(ODD)), dict(q=heads(A * 2, tok=4100)), dict(qo=heads(A * 2, head=132, tok=8192)),
                dict(L=layer(d=96)), dict(rows=(1 << 30) + 1), dict(positions=A + 2), dict(R=rotation(freq=A + 4)),
                dict(positions=None, L=layer(n=[1 << 30], h_kv=1, B=[64]))):
        assert call(lib, norm, **bad) == -2, bad


def test_norm_refusals(lib):
    for bad in (dict(eps=-1e-6), dict(eps=math.nan), dict(eps=math.inf), dict(qw=None), dict(kw=None)):
        assert call(lib, True, **bad) == -1, bad
    assert call(lib, True, q=None, qo=None, qw=None) == 0
    assert call(lib, True, k=None, ko=None, kw=None) == 0
    assert call(lib, True, qw=ODD) == -2


def test_a_single_token_or_head_cannot_meet_itself(lib):
    L = layer(h_q=1, h_kv=1, B=[160])
    assert call(lib, L=L, rows=0, q=heads(tok=128), qo=heads(A * 2, 128, 128), k=heads(tok=128), ko=heads(A * 2, 128, 128)) == 0


def test_frequencies(lib):
    for dims in (2, 4, 20, 64, 128):
        for kw in (dict(), dict(base=500000.0), dict(scaling="linear", factor=4.0), dict(scaling="base", factor=8.0),
                   dict(scaling="parts", factor=8.0, original_len=8192, low=1.0, high=4.0),
                   dict(scaling="parts", factor=32.0, original_len=100, low=0.0, high=0.5), dict(scaling="linear")):
            got, want = np.array(adakv.rotary_frequencies(dims, **kw)), R.frequencies(dims, **kw)
            assert got.shape == (dims // 2,)
            # each is a power of a double, with a few roundings beside it: 16 units in the last place at most, and the
            # exponent's own half unit times ln(base) < 30
            assert np.abs(got / want - 1).max() < 64 * 2.0 ** -53, (dims, kw)


def test_frequency_refusals(lib):
    for bad in (dict(dims=0), dict(dims=3), dict(dims=-2), dict(base=0.0), dict(base=-1.0), dict(base=math.inf), dict(base=math.nan),
                dict(scaling="linear", factor=0.5), dict(scaling="base", factor=math.nan), dict(scaling="base", factor=math.inf),
                dict(scaling="base", base=1e300, factor=1e300), dict(scaling="parts", factor=2.0),
                dict(scaling="parts", factor=2.0, original_len=100, low=2.0, high=2.0),
                dict(scaling="parts", factor=2.0, original_len=100, low=-1.0), dict(scaling="parts", factor=2.0, original_len=100, high=math.inf)):
        with pytest.raises(adakv.AdaKVError) as e:
            adakv.rotary_frequencies(**{**dict(dims=8), **bad})
        assert e.value.status == -1, bad
    with pytest.raises(adakv.AdaKVError) as e:
        adakv.rotary_frequencies(130)
    assert e.value.status == -2
    with pytest.raises(ValueError):
        adakv.rotary_frequencies(64, scaling="other")
    assert lib.adakv_rotary_frequencies(8, 1e4, 4, 1.0, 0, 0.0, 1.0, (ctypes.c_double * 4)()) == -1
    assert lib.adakv_rotary_frequencies(8, 1e4, 0, 1.0, 0, 0.0, 1.0, None) == -1


def test_rotary_arguments(lib):
    for bad in (dict(layout="other"), dict(magnitude=0.0), dict(magnitude=-1.0), dict(scaling="other")):
        with pytest.raises(ValueError):
            adakv.Rotary(64, device="cpu", **bad)
    with pytest.raises(ValueError, match="device tensor"):
        adakv.Rotary(64, device="cpu")
    with pytest.raises(ValueError, match="freq"):
        adakv.Rotary(64, freq=torch.zeros(31, dtype=torch.float64))
    none = adakv.Rotary(0, device="cpu")
    L = layer()
    q, k = torch.zeros(4128, 32, 128, dtype=torch.bfloat16), torch.zeros(4128, 8, 128, dtype=torch.bfloat16)
    for what, a in (("device tensor", dict(q=q, k=k)), ("q or k", dict(q=None, k=None)), ("without q", dict(q=None, k=k, q_out=q)),
                    ("tokens", dict(q=q[:4127], k=k)), ("contiguous rows", dict(q=q[:, :31], k=k)),
                    ("contiguous rows", dict(q=q.transpose(1, 2), k=k)), ("positions", dict(q=q, k=k, positions=torch.zeros(4127, dtype=torch.int32))),
                    ("positions", dict(q=q[:5], k=k[:4], positions=torch.zeros(5, dtype=torch.int32)))):
        with pytest.raises(ValueError, match=what):
            adakv.rotary(L, none, **a)
    with pytest.raises(ValueError, match="k_weight"):
        adakv.norm_rotary(L, none, None, k, None, None)
    with pytest.raises(ValueError, match="q_weight holds"):
        adakv.norm_rotary(L, none, q, k, torch.zeros(64), torch.zeros(128))


def test_the_oracle_turns_pairs():
    """Against complex numbers; and taken back by the negatives of the frequencies."""
    rng = np.random.default_rng(3)
    x, pos = rng.standard_normal((5, 3, 64)), np.array([0, 1, 7, 100000, 5])
    for layout in ("half", "interleaved"):
        for dims in (64, 20, 2, 0):
            f = R.frequencies(dims, base=100.0) if dims else np.zeros(0)
            y = R.turn(x, pos, f, dims, layout, 1.5)
            a, b = (slice(0, dims // 2), slice(dims // 2, dims)) if layout == "half" else (slice(0, dims, 2), slice(1, dims, 2))
            z = (x[..., a] + 1j * x[..., b]) * 1.5 * np.exp(1j * pos[:, None, None] * f)
            assert np.allclose(y[..., a], z.real, atol=1e-12) and np.allclose(y[..., b], z.imag, atol=1e-12)
            assert np.array_equal(y[..., dims:], x[..., dims:])
            assert np.allclose(R.turn(y, pos, -f, dims, layout, 1 / 1.5), x, atol=1e-12)
    y = R.norm(x, np.full(64, 2.0), 0.0)
    assert np.allclose((y ** 2).mean(-1), 4.0)

"""A call on a given stream makes what it is not given (workspace, results) of that stream's memory: the allocator may hand a
block of the current stream's to the next tensor there while the given stream still writes to it, or give one that the
current stream still reads."""
import contextlib

import pytest
import torch

import paper_2407_11550_amd as adakv
from paper_2407_11550_amd import binding

BF = torch.bfloat16
H_Q, H, D, W, HR = 8, 2, 64, 4, 3


def calls(dev):
    """(name, call of a stream) for every call that makes tensors; the results come back as a list."""
    g = torch.Generator().manual_seed(3)
    f = lambda *shape: torch.randn(*shape, generator=g).to(BF).to(dev)
    layer = adakv.Layer(BF, H_Q, H, D, W, 3, 0.2, [50, 70], [40, 48])
    tokens, rows = layer.last_token_row, adakv.cache_rows(layer, HR)
    cu = torch.tensor([0, 20, 40, 64, 88], dtype=torch.int32, device=dev)
    lens = torch.tensor([20, 20, 24, 24], dtype=torch.int32, device=dev)
    budgets = torch.tensor([16, 16, 20, 20], dtype=torch.int32, device=dev)     # (cu: their running sum with the window rows)
    idx = torch.cat([torch.arange(n, dtype=torch.int32) for n in (20, 20, 24, 24)]).to(dev)
    q, K, V, qw = f(tokens, H_Q, D), f(tokens, H, D), f(tokens, H, D), f(2, H_Q, W, D)
    qn, kn, vn, Kc, Vc = f(2, H_Q, D), f(2, H, D), f(2, H, D), f(rows, D), f(rows, D)
    scores = torch.rand(layer.num_scores, generator=g).to(dev)
    q8 = adakv.q8_cache(layer, HR, dev)

    def c(s, *tensors):                          # copies, made where they are used
        with contextlib.nullcontext() if s is None else torch.cuda.stream(s):
            return [type(t)(*(x.clone() for x in t)) if isinstance(t, tuple) else t.clone() for t in tensors]

    step = lambda s, **kw: adakv.decode_step(layer, qn, kn, vn, cu, HR, *c(s, Kc, Vc, lens), want_lse=True, stream=s, **kw)
    return {
        "score": lambda s: adakv.score(layer, qw, K, stream=s),
        "allocate": lambda s: adakv.allocate(layer, scores, stream=s),
        "select": lambda s: adakv.select(layer, scores, budgets, cu, stream=s),
        "compact": lambda s: adakv.compact(layer, K, V, idx, cu, stream=s),
        "compress": lambda s: list(adakv.compress(layer, qw, K, V, stream=s).values()),
        "compress, four calls": lambda s: list(adakv.compress(layer, qw, K, V, stream=s, pipeline=False).values()),
        "compress_static": lambda s: list(adakv.compress_static(layer, qw, K, V, stream=s).values()),
        "probe_read": lambda s: adakv.probe_read(K, stream=s),
        "cache_build": lambda s: adakv.cache_build(layer, K, V, idx, cu, 0, stream=s),
        "decode_attn": lambda s: adakv.decode_attn(layer, qn, cu, HR, Kc, Vc, lens, want_lse=True, stream=s),
        "decode_attn, window": lambda s: adakv.decode_attn(layer, qn, cu, HR, Kc, Vc, lens, want_lse=True, stream=s, window=9, sinks=1),
        "decode_step": step,
        "decode_step, window": lambda s: step(s, window=9, sinks=1),
        "window_attn": lambda s: adakv.window_attn(layer, q, K, V, 9, 1, want_lse=True, stream=s),
        "cache_build_q8": lambda s: adakv.cache_build_q8(layer, K, V, idx, cu, HR, stream=s),
        "decode_attn_q8": lambda s: adakv.decode_attn_q8(layer, qn, cu, HR, q8, lens, want_lse=True, stream=s),
        "decode_step_q8": lambda s: adakv.decode_step_q8(layer, qn, kn, vn, cu, HR, *c(s, q8, lens), want_lse=True, stream=s),
        "cache_move": lambda s: adakv.cache_move(layer, [1, 0], cu, HR, Kc, Vc, lens, HR, stream=s)[1:],
        "cache_move_q8": lambda s: adakv.cache_move_q8(layer, [1, 0], cu, HR, q8, lens, HR, stream=s)[1:],
    }


NAMES = list(calls("cpu"))


def record(monkeypatch, current):
    """Which stream was the current one whenever a call made a tensor."""
    made = []
    for fn in ("empty", "zeros"):
        def make(*a, _fn=getattr(torch, fn), **kw):
            made.append(current())
            return _fn(*a, **kw)
        monkeypatch.setattr(binding.torch, fn, make)
    return made


@pytest.mark.parametrize("name", NAMES)
def test_memory_is_made_on_the_given_stream(name, lib, monkeypatch):
    """(host tensors are refused, after the memory was made)"""
    import types
    call, active, side = calls("cpu")[name], [None], types.SimpleNamespace(device=torch.device("cuda", 0), cuda_stream=7)

    @contextlib.contextmanager
    def stream(s):
        active.append(s)
        yield
        active.pop()

    monkeypatch.setattr(binding.torch.cuda, "stream", stream)
    monkeypatch.setattr(binding, "_device", lambda s: 0)
    monkeypatch.setattr(binding, "_stream", lambda s: 7)
    empty = torch.empty
    monkeypatch.setattr(binding.torch, "empty", lambda *a, **kw: empty(*a, **{**kw, "device": "cpu"}))     # (a workspace is made on the GPU)
    made = record(monkeypatch, lambda: active[-1])
    with pytest.raises(ValueError, match="device tensor"):
        call(side)
    assert made and all(s is side for s in made)
    del made[:]
    with pytest.raises(ValueError, match="device tensor"):
        call(None)
    assert made and all(s is None for s in made)


def leaves(x):
    for t in x if isinstance(x, (tuple, list)) else [x]:
        yield from (leaves(t) if isinstance(t, (tuple, list)) else [t])


@pytest.mark.gpu
@pytest.mark.parametrize("name", NAMES)
def test_the_same_result_on_a_stream_of_its_own(name, monkeypatch):
    """... with both streams' memory filled with NaN before, and with the results let go and the blocks taken again in between."""
    call = calls("cuda:0")[name]
    want = [t.clone() for t in leaves(call(None))]
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    for s in (torch.cuda.current_stream(), side):
        with torch.cuda.stream(s):
            junk = [torch.full((1 << k,), float("nan"), device="cuda:0") for k in range(6, 21)]
            del junk
    torch.cuda.synchronize()
    made = record(monkeypatch, lambda: torch.cuda.current_stream().cuda_stream)
    results = []
    for _ in range(4):
        got = call(side)
        with torch.cuda.stream(side):            # (the copies behind the call, on its stream)
            results.append([t.clone() for t in leaves(got)])
        del got
        torch.full((1 << 18,), float("nan"), device="cuda:0")
    side.synchronize()
    monkeypatch.undo()
    assert made and all(s == side.cuda_stream for s in made)
    for r in results:
        assert len(r) == len(want)
        for x, y in zip(r, want):
            assert torch.equal(x.contiguous().view(torch.uint8), y.contiguous().view(torch.uint8))

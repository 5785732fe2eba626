"""The native checks of the calls around a served cache: what passes them gives what the checks in Python give, and what
does not is left to those."""
import pytest
import torch

import paper_2407_11550_amd as adakv
from paper_2407_11550_amd import binding

BF = torch.bfloat16
H_Q, H, D, W, HR = 8, 2, 64, 4, 3


def arguments(name, dev):
    g = torch.Generator().manual_seed(3)
    f = lambda *shape: torch.randn(*shape, generator=g).to(BF).to(dev)
    i = lambda *v: torch.tensor(v, dtype=torch.int32, device=dev)
    layer = adakv.Layer(BF, H_Q, H, D, W, 3, 0.2, [50, 70], [40, 48])
    tokens, rows = layer.last_token_row, adakv.cache_rows(layer, HR)
    cu, lens = i(0, 20, 40, 64, 88), i(20, 20, 24, 24)
    step = dict(q_new=f(2, H_Q, D), k_new=f(2, H, D), v_new=f(2, H, D), cu_seqlens=cu, headroom=HR)
    rest = dict(seg_len=lens, overflow=i(0), out=torch.zeros(2, H_Q, D, device=dev), lse=torch.zeros(2, H_Q, device=dev),
                ws=torch.zeros(adakv.decode_workspace_bytes(layer, HR), dtype=torch.uint8, device=dev))
    q8 = adakv.q8_cache(layer, HR, dev)
    if name == "decode_step":
        return layer, dict(step, K_cache=f(rows, D), V_cache=f(rows, D), **rest, window=7, sinks=2)
    if name == "decode_step_q8":
        return layer, dict(step, cache=q8, **rest)
    K, V = f(tokens, H, D), f(tokens, H, D)
    if name.startswith("cache_move"):
        to = layer.pick([1, 1, 0])
        more = dict(len_out=i(*[0] * 6), overflow=i(0))
        front = dict(picks=[1, 1, 0], cu_seqlens=cu, headroom=HR)
        if name == "cache_move_q8":
            return layer, dict(front, cache=q8, seg_len=lens, headroom_out=9, cu_out=i(*[0] * 7), out=adakv.q8_cache(to, 9, dev), **more)
        rows_out = adakv.cache_rows(to, 9)
        return layer, dict(front, K_cache=f(rows, D), V_cache=f(rows, D), seg_len=lens, headroom_out=9, cu_out=i(*[0] * 7),
                           K_out=f(rows_out, D), V_out=f(rows_out, D), **more)
    if name == "cache_build_q8":
        idx = torch.cat([torch.arange(n, dtype=torch.int32) for n in (20, 20, 24, 24)]).to(dev)
        return layer, dict(K=K, V=V, indices=idx, cu_seqlens=cu, headroom=HR, cache=q8, seg_len=lens)
    return layer, dict(q=f(tokens, H_Q, D), K=K, V=V, window=9, sinks=1, out=f(tokens, H_Q, D), row_lse=torch.zeros(2, H_Q, W, device=dev))


NAMES = ("decode_step", "decode_step_q8", "cache_build_q8", "window_attn", "cache_move", "cache_move_q8")
strided = lambda t: torch.stack([t, t], dim=-1)[..., 0]


def spoiled(a):
    """(what, arguments) with one argument each not as it has to be: short, of another type, with gaps."""
    for k, v in a.items():
        if isinstance(v, adakv.Q8Cache):
            for part in v._fields:
                t = getattr(v, part)
                yield f"{part} short", dict(a, **{k: v._replace(**{part: t[:-1]})})
                yield f"{part} type", dict(a, **{k: v._replace(**{part: t.view(torch.uint8)})})
        elif isinstance(v, torch.Tensor):
            if k != "ws":
                yield f"{k} short", dict(a, **{k: v[:-1]})
            yield f"{k} type", dict(a, **{k: v.to(torch.float64)})
            if v.numel() > 1:                    # (one element has no gaps)
                yield f"{k} with gaps", dict(a, **{k: strided(v)})
        elif k == "headroom":
            yield "headroom", dict(a, headroom=HR + 1)
        elif k == "headroom_out":
            yield "headroom_out", dict(a, headroom_out=10)
        elif k == "picks":
            yield "picks of no sequence", dict(a, picks=[1, 2, 0])
            yield "no picks", dict(a, picks=[])


def leaves(x):                              # (a picked layer, its numbers)
    for t in x if isinstance(x, (tuple, list)) else [x]:
        yield from (leaves(t) if isinstance(t, (tuple, list)) else [t])


@pytest.mark.parametrize("name", NAMES)
def test_host_tensors_are_left_to_python(name, lib, monkeypatch):
    layer, a = arguments(name, "cpu")
    monkeypatch.setattr(binding, "_device", lambda stream: 0)
    monkeypatch.setattr(binding, "_stream", lambda stream: 7)
    with pytest.raises(ValueError, match="device tensor"):
        getattr(adakv, name)(layer, **a)


def test_wrong_argument_counts(lib):
    for name in ("decode_window_step", "decode_step_q8", "cache_build_q8", "window_attn", "cache_move"):
        with pytest.raises(TypeError, match="takes"):
            getattr(binding._marshal, name)(1, 2)


@pytest.mark.gpu
@pytest.mark.parametrize("name", NAMES)
@pytest.mark.parametrize("without", [(), ("overflow", "lse", "row_lse")])
def test_both_checks_make_the_same_call(name, without, monkeypatch):
    results = []
    for native in (True, False):
        layer, a = arguments(name, "cuda:0")
        a.update({k: None for k in without if k in a})
        calls = []
        if native:
            native_fn = binding._native
            monkeypatch.setattr(binding, "_native", lambda *args, **kw: calls.append(native_fn(*args, **kw)) or calls[-1])
        else:
            monkeypatch.setattr(binding, "_marshal", None)
        out = getattr(adakv, name)(layer, **a)
        torch.cuda.synchronize()
        assert not native or calls == [True]
        monkeypatch.undo()
        results.append([t.clone() for t in leaves(list(a.values()) + [out]) if isinstance(t, torch.Tensor)])
    assert len(results[0]) == len(results[1])
    for x, y in zip(*results):
        assert torch.equal(x.contiguous().view(torch.uint8), y.contiguous().view(torch.uint8))


@pytest.mark.gpu
@pytest.mark.parametrize("name", NAMES)
def test_spoiled_arguments_are_refused_as_in_python(name, monkeypatch):
    layer, good = arguments(name, "cuda:0")
    for what, a in spoiled(good):
        print(what, flush=True)
        said = []
        for native in (True, False):
            with monkeypatch.context() as m:
                if not native:
                    m.setattr(binding, "_marshal", None)
                with pytest.raises((ValueError, adakv.AdaKVError)) as e:
                    getattr(adakv, name)(layer, **a)
                said.append(str(e.value))
        assert said[0] == said[1], what
    torch.cuda.synchronize()

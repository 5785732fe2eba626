"""ctypes binding of libadakv.so: argument marshalling only.

Every step of the path runs in the HIP kernels behind the C ABI (include/adakv.h).
PyTorch is used for device memory and for the stream handle, nothing else.  There is
no fallback: if the library is missing, calls raise.
"""
from __future__ import annotations

import ctypes
import importlib.machinery
import importlib.util
import itertools
import os
from typing import NamedTuple

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
_LIB_PATH = os.path.join(_HERE, "lib", "libadakv.so")
_MARSHAL_PATH = os.path.join(_HERE, "lib", "_marshal.so")
_lib = None
_decode_step_address = 0
_addresses = {}             # of the library's other functions that are called through the native checks

ADAKV_BF16, ADAKV_FP32, ADAKV_FP16 = 0, 1, 2
ADAKV_FLAG_PIPELINE = 2
ADAKV_FLAG_POOL_THEN_MEAN = 4
MAX_BATCH = 64


class AdaKVError(RuntimeError):
    def __init__(self, status, where):
        self.status = status
        msg = load_library().adakv_strerror(status).decode()
        super().__init__(f"{where}: {msg} (status {status})")


class _CLayer(ctypes.Structure):
    _fields_ = [
        ("dtype", ctypes.c_int32), ("h_q", ctypes.c_int32), ("h_kv", ctypes.c_int32),
        ("d", ctypes.c_int32), ("w", ctypes.c_int32), ("pool_k", ctypes.c_int32),
        ("alpha", ctypes.c_float), ("scale", ctypes.c_float), ("batch", ctypes.c_int32),
        ("n", ctypes.POINTER(ctypes.c_int32)), ("B", ctypes.POINTER(ctypes.c_int32)),
        ("tok_off", ctypes.POINTER(ctypes.c_int64)),
        ("k_stride_tok", ctypes.c_int64), ("k_stride_head", ctypes.c_int64),
        ("v_stride_tok", ctypes.c_int64), ("v_stride_head", ctypes.c_int64),
        ("flags", ctypes.c_uint32),
    ]


def library_path() -> str:
    return _LIB_PATH


def load_library():
    """Load libadakv.so (built by __graft_entry__.build()).  Raises if it is not there."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(_LIB_PATH):
        raise RuntimeError(f"{_LIB_PATH} is missing: build it first "
                           "(python -c 'import __graft_entry__ as g; g.build()'); "
                           "there is no fallback path")
    lib = ctypes.CDLL(_LIB_PATH)
    P, V, Z = ctypes.POINTER(_CLayer), ctypes.c_void_p, ctypes.c_size_t
    lib.adakv_workspace_bytes.restype = Z
    lib.adakv_workspace_bytes.argtypes = [P]
    lib.adakv_strerror.restype = ctypes.c_char_p
    lib.adakv_strerror.argtypes = [ctypes.c_int]
    for name, args in (("adakv_score", [P, V, V, V, V, V, Z, V]),
                       ("adakv_allocate", [P, V, V, V, V, Z, V]),
                       ("adakv_select", [P, V, V, V, V, V, Z, V]),
                       ("adakv_compact", [P, V, V, V, V, V, V, V])):
        fn = getattr(lib, name)
        fn.restype = ctypes.c_int
        fn.argtypes = args
    lib.adakv_compress.restype = ctypes.c_int
    lib.adakv_compress.argtypes = [P, V, V, V, V, V, V, V, V, V, V, V, Z, V]
    lib.adakv_compress_static.restype = ctypes.c_int
    lib.adakv_compress_static.argtypes = [P, V, V, V, V, V, V, V, V, V, V, V]
    I = ctypes.c_int32
    for name, args in (("adakv_cache_build", [P, V, V, V, V, I, V, V, V, V]),
                       ("adakv_append", [P, V, V, V, I, V, V, V, V, V]),
                       ("adakv_decode_attn", [P, V, V, I, V, V, V, V, V, V, Z, V]),
                       ("adakv_decode_step", [P, V, V, V, V, I, V, V, V, V, V, V, V, Z, V])):
        fn = getattr(lib, name)
        fn.restype = ctypes.c_int
        fn.argtypes = args
    L64 = ctypes.c_int64
    for name, args in (("adakv_window_attn", [P, V, L64, L64, V, V, I, I, V, V, V]),
                       ("adakv_decode_window_attn", [P, V, V, I, V, V, V, I, I, V, V, V, Z, V]),
                       ("adakv_decode_window_step", [P, V, V, V, V, I, V, V, V, V, I, I, V, V, V, Z, V]),
                       ("adakv_cache_build_q8", [P, V, V, V, V, I, V, V, V, V, V, V]),
                       ("adakv_append_q8", [P, V, V, V, I, V, V, V, V, V, V, V]),
                       ("adakv_decode_attn_q8", [P, V, V, I, V, V, V, V, V, V, V, V, Z, V]),
                       ("adakv_decode_step_q8", [P, V, V, V, V, I, V, V, V, V, V, V, V, V, V, Z, V]),
                       ("adakv_cache_move", [P, I, V, V, I, V, V, V, I, V, V, V, V, V, V]),
                       ("adakv_cache_move_q8", [P, I, V, V, I, V, V, V, V, V, I, V, V, V, V, V, V, V, V])):
        fn = getattr(lib, name)
        fn.restype = ctypes.c_int
        fn.argtypes = args
    lib.adakv_q8_scales.restype = Z
    lib.adakv_q8_scales.argtypes = [P, I]
    lib.adakv_decode_workspace_bytes.restype = Z
    lib.adakv_decode_workspace_bytes.argtypes = [P, I]
    lib.adakv_pyramid_budgets.restype = ctypes.c_int
    lib.adakv_pyramid_budgets.argtypes = [ctypes.c_int32, ctypes.c_int64, ctypes.c_double,
                                          ctypes.POINTER(ctypes.c_int64)]
    lib.adakv_trace_arm.restype = ctypes.c_int
    lib.adakv_trace_arm.argtypes = [ctypes.POINTER(ctypes.c_void_p), ctypes.c_int]
    lib.adakv_trace_disarm.restype = ctypes.c_int
    lib.adakv_trace_disarm.argtypes = []
    lib.adakv_trace_name.restype = ctypes.c_char_p
    lib.adakv_trace_name.argtypes = [ctypes.c_int]
    lib.adakv_describe.restype = ctypes.c_int
    lib.adakv_describe.argtypes = [P, ctypes.c_int, ctypes.c_char_p, Z]
    lib.adakv_probe_read.restype = ctypes.c_int
    lib.adakv_probe_read.argtypes = [V, Z, V, V]
    global _decode_step_address, _marshal
    if _marshal is None:                # built since this module was imported
        _marshal = _load_marshal()
    _decode_step_address = ctypes.cast(lib.adakv_decode_step, V).value
    for name in ("decode_window_step", "decode_step_q8", "cache_build_q8", "window_attn", "cache_move", "cache_move_q8"):
        _addresses[name] = ctypes.cast(getattr(lib, "adakv_" + name), V).value
    _lib = lib
    return lib


class Layer:
    """Host-side description of one layer's compression problem (adakv_layer)."""

    def __init__(self, dtype, h_q, h_kv, d, w, pool_k, alpha, n, B, tok_off=None, scale=0.0,
                 k_strides=None, v_strides=None, flags=0):
        self.torch_dtype = dtype
        self.h_q, self.h_kv, self.d, self.w, self.pool_k = h_q, h_kv, d, w, pool_k
        self.alpha, self.scale = float(alpha), float(scale)
        self.n = [int(v) for v in (n if isinstance(n, (list, tuple)) else [n])]
        self.B = [int(v) for v in (B if isinstance(B, (list, tuple)) else [B])]
        self.batch = len(self.n)
        if tok_off is None:
            tok_off = [0]
            for nb in self.n:
                tok_off.append(tok_off[-1] + nb + w)
        self.tok_off = [int(v) for v in tok_off]
        # of the arrays handed to the library
        self._rows_out, self._segments, self._scores = sum(self.B), self.batch * h_kv, h_kv * sum(self.n)
        self._last_row = None
        self._n = (ctypes.c_int32 * self.batch)(*self.n)
        self._B = (ctypes.c_int32 * len(self.B))(*self.B)
        self._off = (ctypes.c_int64 * len(self.tok_off))(*self.tok_off)
        ks = k_strides or (h_kv * d, d)
        vs = v_strides or (h_kv * d, d)
        self.k_strides, self.v_strides = tuple(int(v) for v in ks), tuple(int(v) for v in vs)
        self.strides_given = (k_strides is not None, v_strides is not None)
        code = {torch.bfloat16: ADAKV_BF16, torch.float32: ADAKV_FP32, torch.float16: ADAKV_FP16}.get(dtype, 99)
        self.c = _CLayer(code, h_q, h_kv, d, w, pool_k, self.alpha, self.scale, self.batch,
                         self._n, self._B, self._off, ks[0], ks[1], vs[0], vs[1], flags)
        self._address = ctypes.addressof(self.c)

    @classmethod
    def from_workload(cls, wl, **kw):
        return cls(wl.dtype, wl.h_q, wl.h_kv, wl.d, wl.w, wl.pool_k, wl.alpha, wl.n, wl.B,
                   tok_off=wl.tok_off, **kw)

    def pick(self, picks) -> "Layer":
        """The layer of a moved cache: its sequence i is this one's sequence picks[i] (its K and V, if it has any, are
        packed one after the other)."""
        if not picks or any(not 0 <= int(b) < self.batch for b in picks):
            raise ValueError(f"picks must name sequences of the layer, 0 to {self.batch - 1}, one at least")
        # (a copy with other sequences: made anew it took longer than moving a small cache)
        new = object.__new__(type(self))
        new.__dict__.update(self.__dict__)
        new.n, new.B = [self.n[b] for b in picks], [self.B[b] for b in picks]
        new.batch = len(new.n)
        new.tok_off = [0, *itertools.accumulate(nb + self.w for nb in new.n)]
        new._rows_out, new._segments, new._scores, new._last_row = sum(new.B), new.batch * self.h_kv, self.h_kv * sum(new.n), None
        new._n, new._B = (ctypes.c_int32 * new.batch)(*new.n), (ctypes.c_int32 * new.batch)(*new.B)
        new._off = (ctypes.c_int64 * (new.batch + 1))(*new.tok_off)
        new.c = _CLayer.from_buffer_copy(self.c)
        new.c.batch, new.c.n, new.c.B, new.c.tok_off = new.batch, new._n, new._B, new._off
        new._address = ctypes.addressof(new.c)
        return new

    @property
    def last_token_row(self):
        """One past the last K/V row any sequence of the layer owns."""
        if self._last_row is None:
            self._last_row = max(self.tok_off[b] + self.n[b] + self.w for b in range(self.batch))
        return self._last_row

    @property
    def num_scores(self):
        return self._scores

    @property
    def num_rows_out(self):
        return self._rows_out

    @property
    def num_segments(self):
        return self._segments


def workspace_bytes(layer: Layer) -> int:
    return int(load_library().adakv_workspace_bytes(ctypes.byref(layer.c)))


def _load_marshal():
    """The module with a decoding step's checks in native code, or None: where it is not built, or was built for
    another torch, the checks here do the same at 5 us more per call."""
    if not os.path.exists(_MARSHAL_PATH):
        return None
    loader = importlib.machinery.ExtensionFileLoader("_marshal", _MARSHAL_PATH)
    try:
        mod = importlib.util.module_from_spec(importlib.util.spec_from_file_location("_marshal", _MARSHAL_PATH, loader=loader))
        loader.exec_module(mod)
    except ImportError:
        return None
    return mod if mod.TORCH_VERSION == torch.__version__.split("+")[0] else None


_marshal = _load_marshal()


def _ptr(t, name, dtype=None):
    if t is None:
        return None
    if not t.is_cuda:
        raise ValueError(f"{name} must be a device tensor")
    if dtype is not None and t.dtype != dtype:
        raise ValueError(f"{name} must be {dtype}, got {t.dtype}")
    return t.data_ptr()                 # (an int: the argument types of the library's functions convert it)


def _need(t, numel, name):
    """A caller-supplied buffer must hold at least `numel` elements, one behind the other (the kernels
    index it by the layer's sizes and never look at the tensor)."""
    if t is None:
        return
    if t.numel() < numel:
        raise ValueError(f"{name} holds {t.numel()} elements, the layer needs {numel}")
    if not t.is_contiguous() and not _dense(t, numel):
        raise ValueError(f"{name} must be contiguous")


def _dense(t, numel):
    """Whether a view's first `numel` elements (the last dimension runs fastest) lie one behind the other."""
    run = 1
    for size, stride in zip(reversed(t.shape), reversed(t.stride())):
        if run >= numel:
            break
        if size != 1 and stride != run:
            return False
        run *= size
    return True


def _check_ws(ws):
    """The workspace's size travels to the library, which checks it."""
    if ws.dtype != torch.uint8:
        raise ValueError("ws must be a uint8 tensor (its size is taken in bytes)")
    if not ws.is_contiguous():
        raise ValueError("ws must be contiguous")


def _check_kv(layer, t, name, strides, given):
    """K or V must cover every row the layer addresses: element offset of the last one read is
    (tok_off[-1] - 1) * stride_tok + (h_kv - 1) * stride_head + d - 1.  When the layer was built
    without explicit strides it assumes a contiguous [tokens, h_kv, d] tensor."""
    if t is None:
        return
    if not given:
        want = (layer.h_kv * layer.d, layer.d, 1)
        if t.dim() != 3 or tuple(t.stride()) != want or t.shape[1] != layer.h_kv or t.shape[2] != layer.d:
            raise ValueError(f"{name} must be a contiguous [tokens, {layer.h_kv}, {layer.d}] tensor "
                             "(or give the Layer its strides)")
    rows = layer.last_token_row
    last = (rows - 1) * strides[0] + (layer.h_kv - 1) * strides[1] + layer.d
    # a view's reachable extent, from its own shape and strides
    extent = 1 + sum((sz - 1) * st for sz, st in zip(t.shape, t.stride())) if t.numel() else 0
    if extent < last:
        raise ValueError(f"{name} reaches {extent} elements from its first one, the layer addresses {last}")


def _native(name, layer, stream, *args, check=None):
    """A call whose arguments are checked in native code.  True: it has been made.  False: something is not as it has to
    be, or is to be made here first, and the checks in Python say what."""
    load_library()
    if _marshal is None:
        return False
    try:
        device, handle = _device(stream), _stream(stream)
    except (RuntimeError, AssertionError, AttributeError):      # no GPU: the tensors are looked at first
        return False
    st = getattr(_marshal, check or name)(device, _addresses[name], layer._address, *args, handle)
    if st is None:
        return False
    if st != 0:
        raise AdaKVError(st, "adakv_" + name)
    return True


def _check_q(layer, q):
    if not q.is_contiguous():
        raise ValueError("q_window must be contiguous")
    _need(q, layer.batch * layer.h_q * layer.w * layer.d, "q_window")


# torch's own functions for the current stream's handle: not part of its public interface, so they may be
# missing in another version
_current_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)
_current_device = getattr(torch._C, "_cuda_getDevice", None)


def _stream(stream):
    """The handle of `stream`, or of the current device's current stream.  A decoding step is two short
    kernels, and making a Stream object for its handle alone took 1.5 of 15 us per call."""
    if stream is None and _current_raw_stream is not None and _current_device is not None:
        return _current_raw_stream(_current_device())
    return (torch.cuda.current_stream() if stream is None else stream).cuda_stream


def _made(make, shape, dtype, device, stream):
    """A tensor that a call on `stream` writes: memory of that stream, which the current one, where the caller may read it,
    is asked about before it is used again."""
    if stream is None:
        return make(shape, dtype=dtype, device=device)
    with torch.cuda.stream(stream):
        t = make(shape, dtype=dtype, device=device)
    if t.is_cuda:
        t.record_stream(torch.cuda.current_stream(t.device))
    return t


def _empty(shape, dtype, device, stream):
    return _made(torch.empty, shape, dtype, device, stream)


def _zeros(shape, dtype, device, stream):
    return _made(torch.zeros, shape, dtype, device, stream)


def _workspace(layer, ws, stream):
    if ws is None:
        ws = _empty(max(workspace_bytes(layer), 16), torch.uint8, "cuda", stream)
    _check_ws(ws)
    return ws, ws.data_ptr(), ws.numel()


def score(layer: Layer, q_window, K, row_lse=None, out=None, ws=None, stream=None):
    """adakv_score: eviction scores [sum_b h_kv*n_b] fp32 (sequence-major, then head)."""
    lib = load_library()
    _check_q(layer, q_window)
    _check_kv(layer, K, "K", layer.k_strides, layer.strides_given[0])
    _need(row_lse, layer.batch * layer.h_q * layer.w, "row_lse")
    if out is None:
        out = _empty(layer._scores, torch.float32, K.device, stream)
    _need(out, layer._scores, "scores")
    ws, wp, wn = _workspace(layer, ws, stream)
    st = lib.adakv_score(ctypes.byref(layer.c), _ptr(q_window, "q_window", layer.torch_dtype),
                         _ptr(K, "K", layer.torch_dtype), _ptr(row_lse, "row_lse", torch.float32),
                         _ptr(out, "scores", torch.float32), wp, wn, _stream(stream))
    if st != 0:
        raise AdaKVError(st, "adakv_score")
    return out


def allocate(layer: Layer, scores, budgets=None, cu_seqlens=None, ws=None, stream=None):
    """adakv_allocate: budgets [batch*h_kv] and cu_seqlens [batch*h_kv+1], int32."""
    lib = load_library()
    if budgets is None:
        budgets = _empty(layer._segments, torch.int32, scores.device, stream)
    if cu_seqlens is None:
        cu_seqlens = _empty(layer._segments + 1, torch.int32, scores.device, stream)
    _need(scores, layer._scores, "scores")
    _need(budgets, layer._segments, "budgets")
    _need(cu_seqlens, layer._segments + 1, "cu_seqlens")
    ws, wp, wn = _workspace(layer, ws, stream)
    st = lib.adakv_allocate(ctypes.byref(layer.c), _ptr(scores, "scores", torch.float32),
                            _ptr(budgets, "budgets", torch.int32),
                            _ptr(cu_seqlens, "cu_seqlens", torch.int32), wp, wn, _stream(stream))
    if st != 0:
        raise AdaKVError(st, "adakv_allocate")
    return budgets, cu_seqlens


def select(layer: Layer, scores, budgets, cu_seqlens, indices=None, ws=None, stream=None):
    """adakv_select: retained positions [sum_b B_b] int32, flattened by (sequence, head)."""
    lib = load_library()
    if indices is None:
        indices = _empty(layer._rows_out, torch.int32, scores.device, stream)
    _need(scores, layer._scores, "scores")
    _need(budgets, layer._segments, "budgets")
    _need(cu_seqlens, layer._segments + 1, "cu_seqlens")
    _need(indices, layer._rows_out, "indices")
    ws, wp, wn = _workspace(layer, ws, stream)
    st = lib.adakv_select(ctypes.byref(layer.c), _ptr(scores, "scores", torch.float32),
                          _ptr(budgets, "budgets", torch.int32),
                          _ptr(cu_seqlens, "cu_seqlens", torch.int32),
                          _ptr(indices, "indices", torch.int32), wp, wn, _stream(stream))
    if st != 0:
        raise AdaKVError(st, "adakv_select")
    return indices


def compact(layer: Layer, K, V, indices, cu_seqlens, K_out=None, V_out=None, stream=None):
    """adakv_compact: K_out, V_out [sum_b B_b, d] in the layer's dtype."""
    lib = load_library()
    if K_out is None:
        K_out = _empty((layer._rows_out, layer.d), layer.torch_dtype, K.device, stream)
    if V_out is None:
        V_out = _empty((layer._rows_out, layer.d), layer.torch_dtype, K.device, stream)
    _check_kv(layer, K, "K", layer.k_strides, layer.strides_given[0])
    _check_kv(layer, V, "V", layer.v_strides, layer.strides_given[1])
    _need(indices, layer._rows_out, "indices")
    _need(cu_seqlens, layer._segments + 1, "cu_seqlens")
    _need(K_out, layer._rows_out * layer.d, "K_out")
    _need(V_out, layer._rows_out * layer.d, "V_out")
    st = lib.adakv_compact(ctypes.byref(layer.c), _ptr(K, "K", layer.torch_dtype),
                           _ptr(V, "V", layer.torch_dtype), _ptr(indices, "indices", torch.int32),
                           _ptr(cu_seqlens, "cu_seqlens", torch.int32),
                           _ptr(K_out, "K_out", layer.torch_dtype),
                           _ptr(V_out, "V_out", layer.torch_dtype), _stream(stream))
    if st != 0:
        raise AdaKVError(st, "adakv_compact")
    return K_out, V_out


def compress(layer: Layer, q_window, K, V, row_lse=None, ws=None, stream=None, bufs=None,
             pipeline=True):
    """The whole step on one stream, no host synchronisation: adakv_compress (one ABI call, pipeline
    mode), or with pipeline=False the four self-contained calls one after the other.
    `bufs` may carry pre-allocated outputs (scores, budgets, cu_seqlens, indices, K_out, V_out)."""
    b = bufs or {}
    dev = K.device
    if ws is None:
        ws = _empty(max(workspace_bytes(layer), 16), torch.uint8, dev, stream)
    if not pipeline:
        sc = score(layer, q_window, K, row_lse=row_lse, out=b.get("scores"), ws=ws, stream=stream)
        bud, cu = allocate(layer, sc, b.get("budgets"), b.get("cu_seqlens"), ws=ws, stream=stream)
        idx = select(layer, sc, bud, cu, b.get("indices"), ws=ws, stream=stream)
        K_out, V_out = compact(layer, K, V, idx, cu, b.get("K_out"), b.get("V_out"), stream=stream)
        return dict(scores=sc, budgets=bud, cu_seqlens=cu, indices=idx, K_out=K_out, V_out=V_out)
    lib = load_library()
    _check_q(layer, q_window)
    _check_kv(layer, K, "K", layer.k_strides, layer.strides_given[0])
    _check_kv(layer, V, "V", layer.v_strides, layer.strides_given[1])
    _need(row_lse, layer.batch * layer.h_q * layer.w, "row_lse")

    def buf(name, shape, dtype):
        t = b.get(name)
        return t if t is not None else _empty(shape, dtype, dev, stream)

    sc = buf("scores", layer._scores, torch.float32)
    bud = buf("budgets", layer._segments, torch.int32)
    cu = buf("cu_seqlens", layer._segments + 1, torch.int32)
    idx = buf("indices", layer._rows_out, torch.int32)
    K_out = buf("K_out", (layer._rows_out, layer.d), layer.torch_dtype)
    V_out = buf("V_out", (layer._rows_out, layer.d), layer.torch_dtype)
    for t, numel, name in ((sc, layer._scores, "scores"), (bud, layer._segments, "budgets"),
                           (cu, layer._segments + 1, "cu_seqlens"), (idx, layer._rows_out, "indices"),
                           (K_out, layer._rows_out * layer.d, "K_out"), (V_out, layer._rows_out * layer.d, "V_out")):
        _need(t, numel, name)
    _check_ws(ws)
    st = lib.adakv_compress(ctypes.byref(layer.c), _ptr(q_window, "q_window", layer.torch_dtype),
                            _ptr(K, "K", layer.torch_dtype), _ptr(V, "V", layer.torch_dtype),
                            _ptr(row_lse, "row_lse", torch.float32), _ptr(sc, "scores", torch.float32),
                            _ptr(bud, "budgets", torch.int32), _ptr(cu, "cu_seqlens", torch.int32),
                            _ptr(idx, "indices", torch.int32), _ptr(K_out, "K_out", layer.torch_dtype),
                            _ptr(V_out, "V_out", layer.torch_dtype), ws.data_ptr(), ws.numel(), _stream(stream))
    if st != 0:
        raise AdaKVError(st, "adakv_compress")
    return dict(scores=sc, budgets=bud, cu_seqlens=cu, indices=idx, K_out=K_out, V_out=V_out)


STATIC_SCRATCH_BYTES = 24 << 20        # ADAKV_STATIC_SCRATCH_BYTES


def compress_static(layer: Layer, q_window, K, V, row_lse=None, stream=None, bufs=None):
    """adakv_compress_static: the whole step with the library's built-in scratch array instead
    of a workspace; the C call allocates nothing (outputs not found in `bufs` are made here)."""
    lib = load_library()
    b = bufs or {}
    dev = K.device
    _check_q(layer, q_window)
    _check_kv(layer, K, "K", layer.k_strides, layer.strides_given[0])
    _check_kv(layer, V, "V", layer.v_strides, layer.strides_given[1])
    _need(row_lse, layer.batch * layer.h_q * layer.w, "row_lse")
    want = (("scores", layer._scores, (layer._scores,), torch.float32),
            ("budgets", layer._segments, (layer._segments,), torch.int32),
            ("cu_seqlens", layer._segments + 1, (layer._segments + 1,), torch.int32),
            ("indices", layer._rows_out, (layer._rows_out,), torch.int32),
            ("K_out", layer._rows_out * layer.d, (layer._rows_out, layer.d), layer.torch_dtype),
            ("V_out", layer._rows_out * layer.d, (layer._rows_out, layer.d), layer.torch_dtype))
    out = {}
    for name, numel, shape, dtype in want:
        t = b.get(name)
        out[name] = t if t is not None else _empty(shape, dtype, dev, stream)
        _need(out[name], numel, name)
    st = lib.adakv_compress_static(
        ctypes.byref(layer.c), _ptr(q_window, "q_window", layer.torch_dtype),
        _ptr(K, "K", layer.torch_dtype), _ptr(V, "V", layer.torch_dtype),
        _ptr(row_lse, "row_lse", torch.float32), _ptr(out["scores"], "scores", torch.float32),
        _ptr(out["budgets"], "budgets", torch.int32), _ptr(out["cu_seqlens"], "cu_seqlens", torch.int32),
        _ptr(out["indices"], "indices", torch.int32), _ptr(out["K_out"], "K_out", layer.torch_dtype),
        _ptr(out["V_out"], "V_out", layer.torch_dtype), _stream(stream))
    if st != 0:
        raise AdaKVError(st, "adakv_compress_static")
    return out


def pyramid_budgets(n_layers: int, avg_budget: int, ratio: float):
    """adakv_pyramid_budgets: per-layer budgets of the pyramidal variant, largest first."""
    out = (ctypes.c_int64 * max(int(n_layers), 1))()
    st = load_library().adakv_pyramid_budgets(int(n_layers), int(avg_budget), float(ratio), out)
    if st != 0:
        raise AdaKVError(st, "adakv_pyramid_budgets")
    return [int(v) for v in out]


def describe(layer: Layer, row_lse: bool = False) -> dict:
    """adakv_describe: the kernel variant a layer of this shape gets, as a dict of its words."""
    buf = ctypes.create_string_buffer(512)
    st = load_library().adakv_describe(ctypes.byref(layer.c), int(bool(row_lse)), buf, 512)
    if st != 0:
        raise AdaKVError(st, "adakv_describe")
    return dict(word.split("=", 1) for word in buf.value.decode().split())


PROBE_SINK_BYTES = 2048 * 4 * 16      # ADAKV_PROBE_SINK_BYTES


def probe_read(src, sink=None, stream=None):
    """adakv_probe_read: one plain streaming read of `src` (a contiguous device tensor whose
    size in bytes is a multiple of 16); returns the sink, one 16-byte XOR word per wave."""
    if not src.is_contiguous():
        raise ValueError("src must be contiguous")
    if sink is None:
        sink = _empty(PROBE_SINK_BYTES, torch.uint8, src.device, stream)
    if sink.numel() * sink.element_size() < PROBE_SINK_BYTES or not sink.is_contiguous():
        raise ValueError("sink too small")
    st = load_library().adakv_probe_read(_ptr(src, "src"), src.numel() * src.element_size(),
                                         _ptr(sink, "sink"), _stream(stream))
    if st != 0:
        raise AdaKVError(st, "adakv_probe_read")
    return sink


# ---- decode side of the flattened layout ---------------------------------------------------------
def cache_rows(layer: Layer, headroom: int) -> int:
    """Rows of K_cache / V_cache: every segment's retained rows plus `headroom` spare rows each."""
    return layer._rows_out + layer._segments * int(headroom)


def _check_cache(layer, headroom, K_cache, V_cache):
    """The cache tensors are addressed as contiguous rows of d elements (a flat tensor of d elements is one row)."""
    for t, name in ((K_cache, "K_cache"), (V_cache, "V_cache")):
        if not t.is_contiguous() or t.size(-1) != layer.d or t.numel() < cache_rows(layer, headroom) * layer.d:
            raise ValueError(f"{name} must be a contiguous [rows, {layer.d}] tensor")


def _check_decode_bufs(layer, headroom, K_cache, V_cache, cu_seqlens, seg_len, out, lse, ws):
    _check_cache(layer, headroom, K_cache, V_cache)
    _need(cu_seqlens, layer._segments + 1, "cu_seqlens")
    _need(seg_len, layer._segments, "seg_len")
    _need(out, layer.batch * layer.h_q * layer.d, "out")
    _need(lse, layer.batch * layer.h_q, "lse")
    _check_ws(ws)


def decode_workspace_bytes(layer: Layer, headroom: int) -> int:
    return int(load_library().adakv_decode_workspace_bytes(ctypes.byref(layer.c), int(headroom)))


def cache_build(layer: Layer, K, V, indices, cu_seqlens, headroom, K_cache=None, V_cache=None,
                seg_len=None, stream=None):
    """adakv_cache_build: the gather of adakv_compact into the layout with head-room; returns
    (K_cache, V_cache, seg_len)."""
    lib = load_library()
    rows = cache_rows(layer, headroom)
    if K_cache is None:
        K_cache = _empty((rows, layer.d), layer.torch_dtype, K.device, stream)
    if V_cache is None:
        V_cache = _empty((rows, layer.d), layer.torch_dtype, K.device, stream)
    if seg_len is None:
        seg_len = _empty(layer._segments, torch.int32, K.device, stream)
    if K_cache.shape[0] < rows or V_cache.shape[0] < rows or seg_len.numel() < layer._segments:
        raise ValueError("cache or seg_len too small for this layer and head-room")
    _check_kv(layer, K, "K", layer.k_strides, layer.strides_given[0])
    _check_kv(layer, V, "V", layer.v_strides, layer.strides_given[1])
    _need(indices, layer._rows_out, "indices")
    _need(cu_seqlens, layer._segments + 1, "cu_seqlens")
    _check_cache(layer, headroom, K_cache, V_cache)
    _need(seg_len, layer._segments, "seg_len")
    st = lib.adakv_cache_build(ctypes.byref(layer.c), _ptr(K, "K", layer.torch_dtype),
                               _ptr(V, "V", layer.torch_dtype), _ptr(indices, "indices", torch.int32),
                               _ptr(cu_seqlens, "cu_seqlens", torch.int32), int(headroom),
                               _ptr(K_cache, "K_cache", layer.torch_dtype),
                               _ptr(V_cache, "V_cache", layer.torch_dtype),
                               _ptr(seg_len, "seg_len", torch.int32), _stream(stream))
    if st != 0:
        raise AdaKVError(st, "adakv_cache_build")
    return K_cache, V_cache, seg_len


def append(layer: Layer, k_new, v_new, cu_seqlens, headroom, K_cache, V_cache, seg_len,
           overflow=None, stream=None):
    """adakv_append: one new K/V row per (sequence, KV head) behind each segment; seg_len grows."""
    lib = load_library()
    want = (layer.batch, layer.h_kv, layer.d)
    if k_new.shape != want or v_new.shape != want:
        raise ValueError(f"k_new and v_new must be {want}")
    if not (k_new.is_contiguous() and v_new.is_contiguous()):
        raise ValueError("k_new and v_new must be contiguous")
    rows = cache_rows(layer, headroom)
    if K_cache.size(0) < rows or V_cache.size(0) < rows:
        raise ValueError("cache too small for this layer and head-room")
    _check_cache(layer, headroom, K_cache, V_cache)
    _need(cu_seqlens, layer._segments + 1, "cu_seqlens")
    _need(seg_len, layer._segments, "seg_len")
    _need(overflow, 1, "overflow")
    st = lib.adakv_append(ctypes.byref(layer.c), _ptr(k_new, "k_new", layer.torch_dtype),
                          _ptr(v_new, "v_new", layer.torch_dtype),
                          _ptr(cu_seqlens, "cu_seqlens", torch.int32), int(headroom),
                          _ptr(K_cache, "K_cache", layer.torch_dtype),
                          _ptr(V_cache, "V_cache", layer.torch_dtype),
                          _ptr(seg_len, "seg_len", torch.int32),
                          _ptr(overflow, "overflow", torch.int32), _stream(stream))
    if st != 0:
        raise AdaKVError(st, "adakv_append")
    return seg_len


def decode_attn(layer: Layer, q_new, cu_seqlens, headroom, K_cache, V_cache, seg_len, out=None,
                lse=None, ws=None, stream=None, want_lse=False, window=None, sinks=0):
    """adakv_decode_attn: out [batch, h_q, d] fp32 (and lse [batch, h_q] if asked for).  With a `window`
    (adakv_decode_window_attn) a segment's last `window` rows and its first `sinks` rows are all that is looked at."""
    window, sinks = _window(window, sinks)
    lib = load_library()
    want = (layer.batch, layer.h_q, layer.d)
    if q_new.shape != want or not q_new.is_contiguous():
        raise ValueError(f"q_new must be contiguous {want}")
    rows = cache_rows(layer, headroom)
    if K_cache.size(0) < rows or V_cache.size(0) < rows:
        raise ValueError("cache too small for this layer and head-room")
    if out is None:
        out = _empty(want, torch.float32, q_new.device, stream)
    if lse is None and want_lse:
        lse = _empty(want[:2], torch.float32, q_new.device, stream)
    if ws is None:
        ws = _empty(max(decode_workspace_bytes(layer, headroom), 16), torch.uint8, q_new.device, stream)
    _check_decode_bufs(layer, headroom, K_cache, V_cache, cu_seqlens, seg_len, out, lse, ws)
    if window is not None:
        _one_device(stream, q_new=q_new, cu_seqlens=cu_seqlens, K_cache=K_cache, V_cache=V_cache, seg_len=seg_len, out=out, lse=lse, ws=ws)
    name, fn = ("adakv_decode_attn", lib.adakv_decode_attn) if window is None else ("adakv_decode_window_attn", lib.adakv_decode_window_attn)
    st = fn(ctypes.byref(layer.c), _ptr(q_new, "q_new", layer.torch_dtype),
            _ptr(cu_seqlens, "cu_seqlens", torch.int32), int(headroom),
            _ptr(K_cache, "K_cache", layer.torch_dtype),
            _ptr(V_cache, "V_cache", layer.torch_dtype),
            _ptr(seg_len, "seg_len", torch.int32), *(() if window is None else (window, sinks)),
            _ptr(out, "out", torch.float32), _ptr(lse, "lse", torch.float32),
            ws.data_ptr(), ws.numel(), _stream(stream))
    if st != 0:
        raise AdaKVError(st, name)
    return (out, lse) if (want_lse or lse is not None) else out


def decode_step(layer: Layer, q_new, k_new, v_new, cu_seqlens, headroom, K_cache, V_cache, seg_len,
                overflow=None, out=None, lse=None, ws=None, stream=None, want_lse=False, window=None, sinks=0):
    """adakv_decode_step: append k_new/v_new to every segment and attend, in one call.  `window`, `sinks`: as for
    decode_attn (adakv_decode_window_step)."""
    lib = load_library()
    window, sinks = _window(window, sinks)
    if window is None and _marshal is not None and out is not None and ws is not None and (lse is not None or not want_lse):
        try:
            handle = _stream(stream)
        except (RuntimeError, AttributeError):      # no GPU, or no stream: the tensors are looked at first
            handle = None
        st = _marshal.decode_step(_decode_step_address, ctypes.addressof(layer.c), q_new, k_new, v_new, cu_seqlens,
                                  headroom, K_cache, V_cache, seg_len, overflow, out, lse, ws, handle)
        if st == 0:
            return out if lse is None else (out, lse)
        if st is not None:
            raise AdaKVError(st, "adakv_decode_step")
        # something is not as it has to be: the checks below say what
    if (window is not None and (lse is not None or not want_lse) and
            _native("decode_window_step", layer, stream, q_new, k_new, v_new, cu_seqlens, headroom, K_cache, V_cache, seg_len, overflow,
                    window, sinks, out, lse, ws)):
        return out if lse is None else (out, lse)
    want = (layer.batch, layer.h_q, layer.d)
    wkv = (layer.batch, layer.h_kv, layer.d)
    if q_new.shape != want or not q_new.is_contiguous():
        raise ValueError(f"q_new must be contiguous {want}")
    if k_new.shape != wkv or v_new.shape != wkv or not (k_new.is_contiguous() and v_new.is_contiguous()):
        raise ValueError(f"k_new and v_new must be contiguous {wkv}")
    rows = cache_rows(layer, headroom)
    if K_cache.size(0) < rows or V_cache.size(0) < rows:
        raise ValueError("cache too small for this layer and head-room")
    if out is None:
        out = _empty(want, torch.float32, q_new.device, stream)
    if lse is None and want_lse:
        lse = _empty(want[:2], torch.float32, q_new.device, stream)
    if ws is None:
        ws = _empty(max(decode_workspace_bytes(layer, headroom), 16), torch.uint8, q_new.device, stream)
    _check_decode_bufs(layer, headroom, K_cache, V_cache, cu_seqlens, seg_len, out, lse, ws)
    _need(overflow, 1, "overflow")
    if window is not None:
        _one_device(stream, q_new=q_new, k_new=k_new, v_new=v_new, cu_seqlens=cu_seqlens, K_cache=K_cache, V_cache=V_cache,
                    seg_len=seg_len, overflow=overflow, out=out, lse=lse, ws=ws)
    name, fn = ("adakv_decode_step", lib.adakv_decode_step) if window is None else ("adakv_decode_window_step", lib.adakv_decode_window_step)
    st = fn(ctypes.byref(layer.c), _ptr(q_new, "q_new", layer.torch_dtype),
            _ptr(k_new, "k_new", layer.torch_dtype),
            _ptr(v_new, "v_new", layer.torch_dtype),
            _ptr(cu_seqlens, "cu_seqlens", torch.int32), int(headroom),
            _ptr(K_cache, "K_cache", layer.torch_dtype),
            _ptr(V_cache, "V_cache", layer.torch_dtype),
            _ptr(seg_len, "seg_len", torch.int32),
            _ptr(overflow, "overflow", torch.int32), *(() if window is None else (window, sinks)),
            _ptr(out, "out", torch.float32), _ptr(lse, "lse", torch.float32),
            ws.data_ptr(), ws.numel(), _stream(stream))
    if st != 0:
        raise AdaKVError(st, name)
    return (out, lse) if (want_lse or lse is not None) else out


# ---- attention over the prompt, limited to a window and sinks -----------------------------------------
def _window(window, sinks):
    """`window` and `sinks` as the library takes them.  A window longer than any sequence means all rows."""
    if window is None:
        if sinks:
            raise ValueError("sinks need a window")
        return None, 0
    window, sinks = int(window), int(sinks)
    if window < 1 or sinks < 0:
        raise ValueError(f"window must be 1 or more and sinks 0 or more, got {window} and {sinks}")
    return min(window, 2**31 - 1), min(sinks, 2**31 - 1)


def _one_device(stream, **tensors):
    """All tensors of a call are on the device that it is launched on: the stream's, or the current one."""
    where = _device(stream)
    for name, t in tensors.items():
        if t is None:
            continue
        if not t.is_cuda:
            raise ValueError(f"{name} must be a device tensor")
        if t.get_device() != where:
            raise ValueError(f"{name} is on device {t.get_device()}, the call is launched on {where}")


def _device(stream):
    if stream is not None:
        return stream.device.index
    return torch.cuda.current_device() if _current_device is None else _current_device()


def window_attn(layer: Layer, q, K, V, window, sinks=0, out=None, row_lse=None, stream=None, want_lse=False):
    """adakv_window_attn: causal attention of q [tokens, h_q, d] (any strides of tokens and heads) over the layer's
    sequences, limited to the last `window` keys and the first `sinks`.  Returns out [tokens, h_q, d] in the layer's
    dtype (rows of no sequence: as they were, zero in an `out` made here) and, if asked for, row_lse [batch, h_q, w] as
    `score` and `compress` take it."""
    lib = load_library()
    window, sinks = _window(window, sinks)
    if window is None:
        raise ValueError("window must be given (the longest sequence's length for all of it)")
    if (row_lse is not None or not want_lse) and _native("window_attn", layer, stream, layer.last_token_row, *layer.strides_given, q, K, V,
                                                         window, sinks, out, row_lse):
        return out if row_lse is None else (out, row_lse)
    if q.dim() != 3 or q.shape[1] != layer.h_q or q.shape[2] != layer.d or (layer.d > 1 and q.stride(2) != 1):
        raise ValueError(f"q must be [tokens, {layer.h_q}, {layer.d}] with contiguous rows")
    rows = layer.last_token_row
    if q.shape[0] < rows:
        raise ValueError(f"q has {q.shape[0]} tokens, the layer's sequences reach {rows}")
    _check_kv(layer, K, "K", layer.k_strides, layer.strides_given[0])
    _check_kv(layer, V, "V", layer.v_strides, layer.strides_given[1])
    if out is None:
        out = _zeros((q.shape[0], layer.h_q, layer.d), layer.torch_dtype, q.device, stream)
    if row_lse is None and want_lse:
        row_lse = _empty((layer.batch, layer.h_q, layer.w), torch.float32, q.device, stream)
    _need(out, rows * layer.h_q * layer.d, "out")
    _need(row_lse, layer.batch * layer.h_q * layer.w, "row_lse")
    dt = layer.torch_dtype
    qp, kp, vp, op, lp = (_ptr(q, "q", dt), _ptr(K, "K", dt), _ptr(V, "V", dt), _ptr(out, "out", dt), _ptr(row_lse, "row_lse", torch.float32))
    _one_device(stream, q=q, K=K, V=V, out=out, row_lse=row_lse)
    st = lib.adakv_window_attn(ctypes.byref(layer.c), qp, q.stride(0), q.stride(1), kp, vp, window, sinks, op, lp, _stream(stream))
    if st != 0:
        raise AdaKVError(st, "adakv_window_attn")
    return (out, row_lse) if (want_lse or row_lse is not None) else out


# ---- the decode-side cache in 8 bits --------------------------------------------------------------------
class Q8Cache(NamedTuple):
    """A cache in 8 bits: K and V [rows, d] torch.float8_e4m3fn, k_scale and v_scale fp32, one for each block of 32 rows
    of a segment (block j of segment s, which starts at row r of the cache: at r // 32 + s + j)."""
    K: torch.Tensor
    V: torch.Tensor
    k_scale: torch.Tensor
    v_scale: torch.Tensor


Q8_BLOCK = 32           # ADAKV_Q8_BLOCK


def q8_scales(layer: Layer, headroom: int) -> int:
    """adakv_q8_scales: how many scales k_scale and v_scale hold."""
    return int(load_library().adakv_q8_scales(ctypes.byref(layer.c), int(headroom)))


def q8_cache(layer: Layer, headroom: int, device="cuda", stream=None) -> Q8Cache:
    """Memory for a cache in 8 bits: zeros (cleared on `stream`, or on the current one)."""
    scales = q8_scales(layer, headroom)
    if scales == 0:
        raise ValueError("the layer or the head-room is not valid")
    codes = [_zeros((cache_rows(layer, headroom), layer.d), torch.uint8, device, stream).view(torch.float8_e4m3fn) for _ in range(2)]
    return Q8Cache(*codes, *(_zeros(scales, torch.float32, device, stream) for _ in range(2)))


def _q8_ptrs(layer, headroom, cache):
    """The four addresses of an 8-bit cache, and its tensors by name."""
    K, V, ks, vs = cache
    _check_cache(layer, headroom, K, V)
    scales = cache_rows(layer, headroom) // Q8_BLOCK + layer._segments
    _need(ks, scales, "k_scale")
    _need(vs, scales, "v_scale")
    f8 = torch.float8_e4m3fn
    return ((_ptr(K, "K", f8), _ptr(V, "V", f8), _ptr(ks, "k_scale", torch.float32), _ptr(vs, "v_scale", torch.float32)),
            dict(K=K, V=V, k_scale=ks, v_scale=vs))


def _check_new(layer, k_new, v_new):
    want = (layer.batch, layer.h_kv, layer.d)
    if k_new.shape != want or v_new.shape != want or not (k_new.is_contiguous() and v_new.is_contiguous()):
        raise ValueError(f"k_new and v_new must be contiguous {want}")


def cache_build_q8(layer: Layer, K, V, indices, cu_seqlens, headroom, cache=None, seg_len=None, stream=None):
    """adakv_cache_build_q8: the gather of cache_build into an 8-bit cache; returns (cache, seg_len)."""
    lib = load_library()
    if cache is not None and _native("cache_build_q8", layer, stream, layer.last_token_row, *layer.strides_given, K, V, indices, cu_seqlens,
                                     headroom, *cache, seg_len):
        return cache, seg_len
    if cache is None:
        cache = q8_cache(layer, headroom, K.device, stream)
    if seg_len is None:
        seg_len = _empty(layer._segments, torch.int32, K.device, stream)
    _check_kv(layer, K, "K", layer.k_strides, layer.strides_given[0])
    _check_kv(layer, V, "V", layer.v_strides, layer.strides_given[1])
    _need(indices, layer._rows_out, "indices")
    _need(cu_seqlens, layer._segments + 1, "cu_seqlens")
    _need(seg_len, layer._segments, "seg_len")
    at, named = _q8_ptrs(layer, headroom, cache)
    args = (_ptr(K, "K", layer.torch_dtype), _ptr(V, "V", layer.torch_dtype), _ptr(indices, "indices", torch.int32),
            _ptr(cu_seqlens, "cu_seqlens", torch.int32), int(headroom), *at, _ptr(seg_len, "seg_len", torch.int32))
    _one_device(stream, K=K, V=V, indices=indices, cu_seqlens=cu_seqlens, seg_len=seg_len, **{"cache." + k: t for k, t in named.items()})
    st = lib.adakv_cache_build_q8(ctypes.byref(layer.c), *args, _stream(stream))
    if st != 0:
        raise AdaKVError(st, "adakv_cache_build_q8")
    return cache, seg_len


def append_q8(layer: Layer, k_new, v_new, cu_seqlens, headroom, cache, seg_len, overflow=None, stream=None):
    """adakv_append_q8: one new K/V row per (sequence, KV head) behind each segment; seg_len grows."""
    lib = load_library()
    _check_new(layer, k_new, v_new)
    _need(cu_seqlens, layer._segments + 1, "cu_seqlens")
    _need(seg_len, layer._segments, "seg_len")
    _need(overflow, 1, "overflow")
    at, named = _q8_ptrs(layer, headroom, cache)
    args = (_ptr(k_new, "k_new", layer.torch_dtype), _ptr(v_new, "v_new", layer.torch_dtype),
            _ptr(cu_seqlens, "cu_seqlens", torch.int32), int(headroom), *at, _ptr(seg_len, "seg_len", torch.int32),
            _ptr(overflow, "overflow", torch.int32))
    _one_device(stream, k_new=k_new, v_new=v_new, cu_seqlens=cu_seqlens, seg_len=seg_len, overflow=overflow, **named)
    st = lib.adakv_append_q8(ctypes.byref(layer.c), *args, _stream(stream))
    if st != 0:
        raise AdaKVError(st, "adakv_append_q8")
    return seg_len


def _decode_q8(name, layer, q_new, new, cu_seqlens, headroom, cache, seg_len, over, out, lse, ws, stream, want_lse):
    """Both decoding calls: `new` and `over` are (k_new, v_new) and (overflow,), or empty."""
    lib = load_library()
    want = (layer.batch, layer.h_q, layer.d)
    if q_new.shape != want or not q_new.is_contiguous():
        raise ValueError(f"q_new must be contiguous {want}")
    if new:
        _check_new(layer, *new)
        _need(over[0], 1, "overflow")
    if out is None:
        out = _empty(want, torch.float32, q_new.device, stream)
    if lse is None and want_lse:
        lse = _empty(want[:2], torch.float32, q_new.device, stream)
    if ws is None:
        ws = _empty(max(decode_workspace_bytes(layer, headroom), 16), torch.uint8, q_new.device, stream)
    at, named = _q8_ptrs(layer, headroom, cache)
    _need(cu_seqlens, layer._segments + 1, "cu_seqlens")
    _need(seg_len, layer._segments, "seg_len")
    _need(out, layer.batch * layer.h_q * layer.d, "out")
    _need(lse, layer.batch * layer.h_q, "lse")
    _check_ws(ws)
    dt = layer.torch_dtype
    args = (_ptr(q_new, "q_new", dt), *(_ptr(t, nm, dt) for t, nm in zip(new, ("k_new", "v_new"))),
            _ptr(cu_seqlens, "cu_seqlens", torch.int32), int(headroom), *at, _ptr(seg_len, "seg_len", torch.int32),
            *(_ptr(t, "overflow", torch.int32) for t in over), _ptr(out, "out", torch.float32), _ptr(lse, "lse", torch.float32))
    _one_device(stream, q_new=q_new, cu_seqlens=cu_seqlens, seg_len=seg_len, out=out, lse=lse, ws=ws, **named,
                **dict(zip(("k_new", "v_new"), new)), **dict(zip(("overflow",), over)))
    st = getattr(lib, name)(ctypes.byref(layer.c), *args, ws.data_ptr(), ws.numel(), _stream(stream))
    if st != 0:
        raise AdaKVError(st, name)
    return (out, lse) if (want_lse or lse is not None) else out


def decode_attn_q8(layer: Layer, q_new, cu_seqlens, headroom, cache, seg_len, out=None, lse=None, ws=None, stream=None, want_lse=False):
    """adakv_decode_attn_q8: decode_attn over an 8-bit cache."""
    return _decode_q8("adakv_decode_attn_q8", layer, q_new, (), cu_seqlens, headroom, cache, seg_len, (), out, lse, ws, stream, want_lse)


def decode_step_q8(layer: Layer, q_new, k_new, v_new, cu_seqlens, headroom, cache, seg_len, overflow=None, out=None, lse=None,
                   ws=None, stream=None, want_lse=False):
    """adakv_decode_step_q8: decode_step over an 8-bit cache."""
    if (lse is not None or not want_lse) and _native("decode_step_q8", layer, stream, q_new, k_new, v_new, cu_seqlens, headroom, *cache,
                                                     seg_len, overflow, out, lse, ws):
        return out if lse is None else (out, lse)
    return _decode_q8("adakv_decode_step_q8", layer, q_new, (k_new, v_new), cu_seqlens, headroom, cache, seg_len, (overflow,), out,
                      lse, ws, stream, want_lse)


# ---- sequences of a cache, moved ------------------------------------------------------------------------
def _move(name, layer, picks, cu_seqlens, headroom, src, seg_len, headroom_out, cu_out, dst, len_out, overflow, stream):
    to = layer.pick(picks)
    _need(cu_seqlens, layer._segments + 1, "cu_seqlens")
    _need(seg_len, layer._segments, "seg_len")
    _need(overflow, 1, "overflow")
    dev = cu_seqlens.device
    if cu_out is None:
        cu_out = _empty(to._segments + 1, torch.int32, dev, stream)
    if len_out is None:
        len_out = _empty(to._segments, torch.int32, dev, stream)
    _need(cu_out, to._segments + 1, "cu_out")
    _need(len_out, to._segments, "len_out")
    (at, named), (at_out, named_out) = src(layer, headroom), dst(to, headroom_out)
    i32 = torch.int32
    args = (len(picks), (ctypes.c_int32 * len(picks))(*(int(b) for b in picks)), _ptr(cu_seqlens, "cu_seqlens", i32), int(headroom), *at,
            _ptr(seg_len, "seg_len", i32), int(headroom_out), _ptr(cu_out, "cu_out", i32), *at_out, _ptr(len_out, "len_out", i32),
            _ptr(overflow, "overflow", i32))
    _one_device(stream, cu_seqlens=cu_seqlens, seg_len=seg_len, cu_out=cu_out, len_out=len_out, overflow=overflow, **named,
                **{k + "_out": t for k, t in named_out.items()})
    st = getattr(load_library(), name)(ctypes.byref(layer.c), *args, _stream(stream))
    if st != 0:
        raise AdaKVError(st, name)
    return to, cu_out, len_out


def cache_move(layer: Layer, picks, cu_seqlens, headroom, K_cache, V_cache, seg_len, headroom_out, cu_out=None, K_out=None,
               V_out=None, len_out=None, overflow=None, stream=None):
    """adakv_cache_move: the cache of sequences picks[0], picks[1], ... (forked where named twice, dropped where not) with
    other head-room.  Returns (layer.pick(picks), cu_out, K_out, V_out, len_out)."""
    def cache(K, V):
        def at(lay, hr):
            _check_cache(lay, hr, K, V)
            return tuple(_ptr(t, nm, lay.torch_dtype) for t, nm in ((K, "K_cache"), (V, "V_cache"))), dict(K=K, V=V)
        return at

    if _native("cache_move", layer, stream, picks, cu_seqlens, headroom, K_cache, V_cache, None, None, seg_len, headroom_out, cu_out, K_out,
               V_out, None, None, len_out, overflow):
        return layer.pick(picks), cu_out, K_out, V_out, len_out
    rows = cache_rows(layer.pick(picks), headroom_out)
    if K_out is None:
        K_out = _zeros((rows, layer.d), layer.torch_dtype, K_cache.device, stream)
    if V_out is None:
        V_out = _zeros((rows, layer.d), layer.torch_dtype, V_cache.device, stream)
    to, cu_out, len_out = _move("adakv_cache_move", layer, picks, cu_seqlens, headroom, cache(K_cache, V_cache), seg_len, headroom_out,
                                cu_out, cache(K_out, V_out), len_out, overflow, stream)
    return to, cu_out, K_out, V_out, len_out


def cache_move_q8(layer: Layer, picks, cu_seqlens, headroom, cache, seg_len, headroom_out, cu_out=None, out=None, len_out=None,
                  overflow=None, stream=None):
    """adakv_cache_move_q8: cache_move for an 8-bit cache.  Returns (layer.pick(picks), cu_out, out, len_out)."""
    if out is not None and _native("cache_move_q8", layer, stream, picks, cu_seqlens, headroom, *cache, seg_len, headroom_out, cu_out, *out,
                                   len_out, overflow, check="cache_move"):
        return layer.pick(picks), cu_out, out, len_out
    if out is None:
        out = q8_cache(layer.pick(picks), headroom_out, cache.K.device, stream)
    to, cu_out, len_out = _move("adakv_cache_move_q8", layer, picks, cu_seqlens, headroom, lambda lay, hr: _q8_ptrs(lay, hr, cache), seg_len,
                                headroom_out, cu_out, lambda lay, hr: _q8_ptrs(lay, hr, out), len_out, overflow, stream)
    return to, cu_out, out, len_out


class KernelTrace:
    """Per-kernel timing through adakv_trace_arm: inside the `with` block every kernel the
    library launches carries a pair of events that receive its own start and end time."""

    def __init__(self, capacity=128):
        self.events = [torch.cuda.Event(enable_timing=True) for _ in range(capacity)]
        for ev in self.events:                      # the first record creates the HIP event
            ev.record()
        self._arr = (ctypes.c_void_p * capacity)(*[ev.cuda_event for ev in self.events])
        self.used = 0
        self.names = []

    def __enter__(self):
        st = load_library().adakv_trace_arm(self._arr, len(self.events))
        if st != 0:
            raise AdaKVError(st, "adakv_trace_arm")
        return self

    def __exit__(self, *exc):
        lib = load_library()
        self.names = [lib.adakv_trace_name(i).decode() for i in range(len(self.events))]
        self.used = lib.adakv_trace_disarm()
        self.names = self.names[:self.used]
        return False

    def durations_us(self):
        """[(kernel name, microseconds)] for every traced kernel; call after a synchronize."""
        return [(self.names[i], 1000.0 * self.events[i].elapsed_time(self.events[i + 1]))
                for i in range(0, self.used - 1, 2)]

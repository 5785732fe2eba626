// The argument checks of the calls whose kernels take less time than these did in Python, in native code, for the binding.
// First of them a decoding step.  A step of a short cache is two kernels of
// 8.6 us together, and the checks of its twelve tensors took 5 us of interpreter time per call, so that the host and
// not the GPU decided how long it took: 11.3 us to issue one, now 6.6, and a step over 8 KV heads of 512 rows at
// d = 64 took 11.0 us, now 9.1.  Only the case in which everything is as it has to be is handled here: whatever is
// not comes back as None, and the checks in binding.py look again and report it.
#include <Python.h>
#include <torch/csrc/autograd/python_variable.h>
#include <torch/version.h>

#include <limits>

#include "adakv.h"

namespace {

typedef int (*StepFn)(const adakv_layer *, const void *, const void *, const void *, const int32_t *, int32_t, void *, void *,
                      int32_t *, int32_t *, float *, float *, void *, size_t, void *);

// A plain tensor on the GPU of the given type, else nullptr (subclasses are the interpreter's business).
const at::Tensor *device_tensor(PyObject *o, at::ScalarType type) {
  if (!THPVariable_CheckExact(o)) return nullptr;
  const at::Tensor &t = THPVariable_Unpack(o);
  return t.is_cuda() && t.scalar_type() == type ? &t : nullptr;
}
bool is_rows(const at::Tensor *t, int64_t batch, int64_t h, int64_t d) {
  return t && t->dim() == 3 && t->size(0) == batch && t->size(1) == h && t->size(2) == d && t->is_contiguous();
}
bool is_cache(const at::Tensor *t, int64_t rows, int64_t d) {
  return t && t->dim() >= 1 && t->size(0) >= rows && t->size(-1) == d && t->numel() >= rows * d && t->is_contiguous();
}
bool holds(const at::Tensor *t, int64_t numel) { return t && t->numel() >= numel && t->is_contiguous(); }

// decode_step(function, layer, q, k, v, cu_seqlens, headroom, K_cache, V_cache, seg_len, overflow, out, lse, ws, stream)
// -> the library's status, or None where the arguments are for binding.py to look at
PyObject *decode_step(PyObject *, PyObject *const *a, Py_ssize_t n) {
  if (n != 15) {
    PyErr_SetString(PyExc_TypeError, "decode_step takes 15 arguments");
    return nullptr;
  }
  const StepFn fn = reinterpret_cast<StepFn>(PyLong_AsVoidPtr(a[0]));
  const adakv_layer *L = static_cast<const adakv_layer *>(PyLong_AsVoidPtr(a[1]));
  void *stream = PyLong_AsVoidPtr(a[14]);
  const long headroom = PyLong_Check(a[6]) ? PyLong_AsLong(a[6]) : -1;
  if (PyErr_Occurred()) {                      // an address, a stream or a head-room that is no whole number
    PyErr_Clear();
    Py_RETURN_NONE;
  }
  if (!fn || !L || headroom < 0 || headroom > std::numeric_limits<int32_t>::max()) Py_RETURN_NONE;
  try {
    const at::ScalarType type = L->dtype == ADAKV_BF16 ? at::kBFloat16 : L->dtype == ADAKV_FP16 ? at::kHalf : at::kFloat;
    if ((L->dtype != ADAKV_FP32 && type == at::kFloat) || L->batch < 1 || L->batch > ADAKV_MAX_BATCH) Py_RETURN_NONE;
    const int64_t nseg = (int64_t)L->batch * L->h_kv;
    int64_t rows = nseg * headroom;
    for (int b = 0; b < L->batch; ++b) rows += L->B[b];
    const at::Tensor *q = device_tensor(a[2], type), *k = device_tensor(a[3], type), *v = device_tensor(a[4], type);
    const at::Tensor *cu = device_tensor(a[5], at::kInt), *Kc = device_tensor(a[7], type), *Vc = device_tensor(a[8], type);
    const at::Tensor *len = device_tensor(a[9], at::kInt), *over = a[10] == Py_None ? nullptr : device_tensor(a[10], at::kInt);
    const at::Tensor *out = device_tensor(a[11], at::kFloat), *lse = a[12] == Py_None ? nullptr : device_tensor(a[12], at::kFloat);
    const at::Tensor *ws = device_tensor(a[13], at::kByte);
    if (!is_rows(q, L->batch, L->h_q, L->d) || !is_rows(k, L->batch, L->h_kv, L->d) || !is_rows(v, L->batch, L->h_kv, L->d) ||
        !is_cache(Kc, rows, L->d) || !is_cache(Vc, rows, L->d) || !holds(cu, nseg + 1) || !holds(len, nseg) ||
        (a[10] != Py_None && !holds(over, 1)) || !holds(out, (int64_t)L->batch * L->h_q * L->d) ||
        (a[12] != Py_None && !holds(lse, (int64_t)L->batch * L->h_q)) || !holds(ws, 0))
      Py_RETURN_NONE;
    void *p[12] = {q->data_ptr(), k->data_ptr(), v->data_ptr(), cu->data_ptr(), Kc->data_ptr(), Vc->data_ptr(), len->data_ptr(),
                   over ? over->data_ptr() : nullptr, out->data_ptr(), lse ? lse->data_ptr() : nullptr, ws->data_ptr(), stream};
    const size_t ws_bytes = (size_t)ws->numel();
    int st;
    Py_BEGIN_ALLOW_THREADS
    st = fn(L, p[0], p[1], p[2], (const int32_t *)p[3], (int32_t)headroom, p[4], p[5], (int32_t *)p[6], (int32_t *)p[7],
            (float *)p[8], (float *)p[9], p[10], ws_bytes, p[11]);
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(st);
  } catch (...) {                              // a tensor without memory of its own, for instance
    Py_RETURN_NONE;
  }
}

// ---- the other calls: as above, and all tensors on the device that the call is launched on --------------------------
struct Refused {};                             // left to binding.py

// Takes a call's Python arguments in order; the first that is not as it has to be ends it.
struct Args {
  PyObject *const *a;
  int at = 0;
  int device = -1;

  long long whole(long long least, long long most) {
    PyObject *o = a[at++];
    if (!PyLong_Check(o)) throw Refused();
    const long long v = PyLong_AsLongLong(o);
    if (PyErr_Occurred() || v < least || v > most) throw Refused();
    return v;
  }
  int32_t i32(long long least = 0) { return (int32_t)whole(least, std::numeric_limits<int32_t>::max()); }
  void *pointer() {
    void *p = PyLong_AsVoidPtr(a[at++]);
    if (PyErr_Occurred()) throw Refused();
    return p;
  }
  const at::Tensor &tensor(at::ScalarType type) {
    const at::Tensor *t = device_tensor(a[at++], type);
    if (!t || t->get_device() != device) throw Refused();
    return *t;
  }
  // one behind the other, so many at least
  const at::Tensor &buffer(at::ScalarType type, int64_t numel) {
    const at::Tensor &t = tensor(type);
    if (!holds(&t, numel)) throw Refused();
    return t;
  }
  template <typename T> T *data(at::ScalarType type, int64_t numel) { return static_cast<T *>(buffer(type, numel).data_ptr()); }
  template <typename T> T *data_or_none(at::ScalarType type, int64_t numel) {
    if (a[at] != Py_None) return data<T>(type, numel);
    ++at;
    return nullptr;
  }
  void *rows(at::ScalarType type, int64_t batch, int64_t h, int64_t d) {
    const at::Tensor &t = tensor(type);
    if (!is_rows(&t, batch, h, d)) throw Refused();
    return t.data_ptr();
  }
  void *cache(at::ScalarType type, int64_t rows, int64_t d) {
    const at::Tensor &t = tensor(type);
    if (!is_cache(&t, rows, d)) throw Refused();
    return t.data_ptr();
  }
  // K or V: strides of the layer, which reach `tokens` rows; `given`: not those of a contiguous tensor
  void *keys(const adakv_layer *L, at::ScalarType type, int64_t tokens, int64_t s_tok, int64_t s_head, bool given) {
    const at::Tensor &t = tensor(type);
    if (!given && !(t.dim() == 3 && t.size(1) == L->h_kv && t.size(2) == L->d && t.stride(0) == (int64_t)L->h_kv * L->d &&
                    t.stride(1) == L->d && t.stride(2) == 1))
      throw Refused();
    int64_t extent = t.numel() ? 1 : 0;
    for (int64_t i = 0; t.numel() && i < t.dim(); ++i) extent += (t.size(i) - 1) * t.stride(i);
    if (extent < (tokens - 1) * s_tok + (L->h_kv - 1) * s_head + L->d) throw Refused();
    return t.data_ptr();
  }
};

// The layer at the front of a call's arguments, and what follows from it.
struct Layer {
  const adakv_layer *L;
  at::ScalarType type;
  int64_t nseg, kept = 0;
  explicit Layer(Args &x) : L(static_cast<const adakv_layer *>(x.pointer())) {
    if (!L || L->batch < 1 || L->batch > ADAKV_MAX_BATCH) throw Refused();
    type = L->dtype == ADAKV_BF16 ? at::kBFloat16 : L->dtype == ADAKV_FP16 ? at::kHalf : at::kFloat;
    if (L->dtype != ADAKV_FP32 && type == at::kFloat) throw Refused();
    nseg = (int64_t)L->batch * L->h_kv;
    for (int b = 0; b < L->batch; ++b) kept += L->B[b];
  }
  int64_t rows(int32_t headroom) const { return kept + nseg * headroom; }
};

template <typename F> PyObject *checked(const char *name, Py_ssize_t n, Py_ssize_t want, PyObject *const *a, F &&call) {
  if (n != want) {
    PyErr_Format(PyExc_TypeError, "%s takes %zd arguments", name, want);
    return nullptr;
  }
  try {
    Args x{a};
    x.device = (int)x.whole(0, 1 << 16);
    return PyLong_FromLong(call(x));
  } catch (...) {                              // Refused, or a tensor without memory of its own
    PyErr_Clear();
    Py_RETURN_NONE;
  }
}

// A call of the library without the interpreter's lock, which is back however the call ends.  `f` asks no tensor for anything:
// what a tensor says may be an exception.
template <typename F> int unlocked(F &&f) {
  struct Unlock {
    PyThreadState *state = PyEval_SaveThread();
    ~Unlock() { PyEval_RestoreThread(state); }
  } unlock;
  return f();
}

// (device, function, layer, q, k, v, cu_seqlens, headroom, K_cache, V_cache, seg_len, overflow, window, sinks, out, lse, ws, stream)
PyObject *decode_window_step(PyObject *, PyObject *const *a, Py_ssize_t n) {
  return checked("decode_window_step", n, 18, a, [](Args &x) {
    const auto fn = reinterpret_cast<decltype(&adakv_decode_window_step)>(x.pointer());
    const Layer l(x);
    const adakv_layer *L = l.L;
    void *q = x.rows(l.type, L->batch, L->h_q, L->d), *k = x.rows(l.type, L->batch, L->h_kv, L->d), *v = x.rows(l.type, L->batch, L->h_kv, L->d);
    const int32_t *cu = x.data<int32_t>(at::kInt, l.nseg + 1);
    const int32_t headroom = x.i32();
    void *K = x.cache(l.type, l.rows(headroom), L->d), *V = x.cache(l.type, l.rows(headroom), L->d);
    int32_t *len = x.data<int32_t>(at::kInt, l.nseg), *over = x.data_or_none<int32_t>(at::kInt, 1);
    const int32_t window = x.i32(1), sinks = x.i32();
    float *out = x.data<float>(at::kFloat, (int64_t)L->batch * L->h_q * L->d), *lse = x.data_or_none<float>(at::kFloat, (int64_t)L->batch * L->h_q);
    const at::Tensor &ws = x.buffer(at::kByte, 0);
    const size_t ws_bytes = (size_t)ws.numel();
    void *p = ws.data_ptr(), *stream = x.pointer();
    return unlocked([&] { return fn(L, q, k, v, cu, headroom, K, V, len, over, window, sinks, out, lse, p, ws_bytes, stream); });
  });
}

// (device, function, layer, q, k, v, cu_seqlens, headroom, K, V, k_scale, v_scale, seg_len, overflow, out, lse, ws, stream)
PyObject *decode_step_q8(PyObject *, PyObject *const *a, Py_ssize_t n) {
  return checked("decode_step_q8", n, 18, a, [](Args &x) {
    const auto fn = reinterpret_cast<decltype(&adakv_decode_step_q8)>(x.pointer());
    const Layer l(x);
    const adakv_layer *L = l.L;
    void *q = x.rows(l.type, L->batch, L->h_q, L->d), *k = x.rows(l.type, L->batch, L->h_kv, L->d), *v = x.rows(l.type, L->batch, L->h_kv, L->d);
    const int32_t *cu = x.data<int32_t>(at::kInt, l.nseg + 1);
    const int32_t headroom = x.i32();
    const int64_t rows = l.rows(headroom), scales = rows / ADAKV_Q8_BLOCK + l.nseg;
    void *K = x.cache(at::kFloat8_e4m3fn, rows, L->d), *V = x.cache(at::kFloat8_e4m3fn, rows, L->d);
    float *ks = x.data<float>(at::kFloat, scales), *vs = x.data<float>(at::kFloat, scales);
    int32_t *len = x.data<int32_t>(at::kInt, l.nseg), *over = x.data_or_none<int32_t>(at::kInt, 1);
    float *out = x.data<float>(at::kFloat, (int64_t)L->batch * L->h_q * L->d), *lse = x.data_or_none<float>(at::kFloat, (int64_t)L->batch * L->h_q);
    const at::Tensor &ws = x.buffer(at::kByte, 0);
    const size_t ws_bytes = (size_t)ws.numel();
    void *p = ws.data_ptr(), *stream = x.pointer();
    return unlocked([&] { return fn(L, q, k, v, cu, headroom, K, V, ks, vs, len, over, out, lse, p, ws_bytes, stream); });
  });
}

// (device, function, layer, tokens, K's strides given, V's, K, V, indices, cu_seqlens, headroom, K_q8, V_q8, k_scale, v_scale, seg_len, stream)
PyObject *cache_build_q8(PyObject *, PyObject *const *a, Py_ssize_t n) {
  return checked("cache_build_q8", n, 17, a, [](Args &x) {
    const auto fn = reinterpret_cast<decltype(&adakv_cache_build_q8)>(x.pointer());
    const Layer l(x);
    const adakv_layer *L = l.L;
    const int64_t tokens = x.whole(1, std::numeric_limits<int64_t>::max());
    const bool kg = x.whole(0, 1) != 0, vg = x.whole(0, 1) != 0;
    void *K = x.keys(L, l.type, tokens, L->k_stride_tok, L->k_stride_head, kg), *V = x.keys(L, l.type, tokens, L->v_stride_tok, L->v_stride_head, vg);
    const int32_t *idx = x.data<int32_t>(at::kInt, l.kept), *cu = x.data<int32_t>(at::kInt, l.nseg + 1);
    const int32_t headroom = x.i32();
    const int64_t rows = l.rows(headroom), scales = rows / ADAKV_Q8_BLOCK + l.nseg;
    void *Kq = x.cache(at::kFloat8_e4m3fn, rows, L->d), *Vq = x.cache(at::kFloat8_e4m3fn, rows, L->d);
    float *ks = x.data<float>(at::kFloat, scales), *vs = x.data<float>(at::kFloat, scales);
    int32_t *len = x.data<int32_t>(at::kInt, l.nseg);
    void *stream = x.pointer();
    return unlocked([&] { return fn(L, K, V, idx, cu, headroom, Kq, Vq, ks, vs, len, stream); });
  });
}

// (device, function, layer, tokens, K's strides given, V's, q, K, V, window, sinks, out, row_lse, stream)
PyObject *window_attn(PyObject *, PyObject *const *a, Py_ssize_t n) {
  return checked("window_attn", n, 14, a, [](Args &x) {
    const auto fn = reinterpret_cast<decltype(&adakv_window_attn)>(x.pointer());
    const Layer l(x);
    const adakv_layer *L = l.L;
    const int64_t tokens = x.whole(1, std::numeric_limits<int64_t>::max());
    const bool kg = x.whole(0, 1) != 0, vg = x.whole(0, 1) != 0;
    const at::Tensor &q = x.tensor(l.type);
    if (q.dim() != 3 || q.size(0) < tokens || q.size(1) != L->h_q || q.size(2) != L->d || q.stride(2) != 1) throw Refused();
    void *K = x.keys(L, l.type, tokens, L->k_stride_tok, L->k_stride_head, kg), *V = x.keys(L, l.type, tokens, L->v_stride_tok, L->v_stride_head, vg);
    const int32_t window = x.i32(1), sinks = x.i32();
    void *out = x.data<void>(l.type, tokens * L->h_q * L->d);
    float *lse = x.data_or_none<float>(at::kFloat, (int64_t)L->batch * L->h_q * L->w);
    void *stream = x.pointer();
    const int64_t q_tok = q.stride(0), q_head = q.stride(1);
    void *qp = q.data_ptr();
    return unlocked([&] { return fn(L, qp, q_tok, q_head, K, V, window, sinks, out, lse, stream); });
  });
}

// (device, function, layer, picks, cu_seqlens, headroom, K, V, k_scale, v_scale, seg_len, headroom_out, cu_out, K_out, V_out, k_scale_out,
// v_scale_out, len_out, overflow, stream); scales of a cache in 8 bits, else None: the function is the one for it
PyObject *cache_move(PyObject *, PyObject *const *a, Py_ssize_t n) {
  return checked("cache_move", n, 20, a, [](Args &x) {
    void *fn = x.pointer();
    const Layer l(x);
    const adakv_layer *L = l.L;
    PyObject *picks = x.a[x.at++];
    if (!PyList_CheckExact(picks) || PyList_GET_SIZE(picks) < 1 || PyList_GET_SIZE(picks) > ADAKV_MAX_BATCH) throw Refused();
    const int32_t count = (int32_t)PyList_GET_SIZE(picks);
    int32_t from[ADAKV_MAX_BATCH];
    int64_t kept = 0;
    for (int32_t i = 0; i < count; ++i) {
      PyObject *o = PyList_GET_ITEM(picks, i);
      const long long b = PyLong_CheckExact(o) ? PyLong_AsLongLong(o) : -1;
      if (PyErr_Occurred() || b < 0 || b >= L->batch) throw Refused();
      from[i] = (int32_t)b;
      kept += L->B[b];
    }
    const int32_t *cu = x.data<int32_t>(at::kInt, l.nseg + 1);
    const bool q8 = x.a[x.at + 3] != Py_None;
    const at::ScalarType type = q8 ? at::kFloat8_e4m3fn : l.type;
    struct { void *K, *V; float *ks, *vs; } c[2];
    int32_t headroom[2], *cu_out = nullptr;
    const int32_t *len = nullptr;
    for (int o = 0; o < 2; ++o) {              // the source, the destination
      const int64_t nseg = o ? (int64_t)count * L->h_kv : l.nseg;
      headroom[o] = x.i32();
      if (o) cu_out = x.data<int32_t>(at::kInt, nseg + 1);
      const int64_t rows = (o ? kept : l.kept) + nseg * headroom[o], scales = rows / ADAKV_Q8_BLOCK + nseg;
      c[o].K = x.cache(type, rows, L->d);
      c[o].V = x.cache(type, rows, L->d);
      c[o].ks = x.data_or_none<float>(at::kFloat, scales);
      c[o].vs = x.data_or_none<float>(at::kFloat, scales);
      if ((c[o].ks != nullptr) != q8 || (c[o].vs != nullptr) != q8) throw Refused();
      if (!o) len = x.data<int32_t>(at::kInt, nseg);
    }
    int32_t *len_out = x.data<int32_t>(at::kInt, (int64_t)count * L->h_kv), *over = x.data_or_none<int32_t>(at::kInt, 1);
    void *stream = x.pointer();
    return unlocked([&] {
      if (q8)
        return reinterpret_cast<decltype(&adakv_cache_move_q8)>(fn)(L, count, from, cu, headroom[0], c[0].K, c[0].V, c[0].ks, c[0].vs, len, headroom[1],
                                                                   cu_out, c[1].K, c[1].V, c[1].ks, c[1].vs, len_out, over, stream);
      return reinterpret_cast<decltype(&adakv_cache_move)>(fn)(L, count, from, cu, headroom[0], c[0].K, c[0].V, len, headroom[1], cu_out, c[1].K,
                                                              c[1].V, len_out, over, stream);
    });
  });
}

PyMethodDef methods[] = {
    {"decode_step", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(decode_step)), METH_FASTCALL,
     "decode_step(function, layer, q, k, v, cu_seqlens, headroom, K_cache, V_cache, seg_len, overflow, out, lse, ws, stream)"},
#define ADAKV_METHOD(name) {#name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(name)), METH_FASTCALL, nullptr}
    ADAKV_METHOD(decode_window_step),
    ADAKV_METHOD(decode_step_q8),
    ADAKV_METHOD(cache_build_q8),
    ADAKV_METHOD(window_attn),
    ADAKV_METHOD(cache_move),
#undef ADAKV_METHOD
    {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_marshal", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

// TORCH_VERSION: a tensor's layout is that of the headers compiled against, which binding.py compares with torch itself.
PyMODINIT_FUNC PyInit__marshal() {
  PyObject *m = PyModule_Create(&module);
  if (m && PyModule_AddStringConstant(m, "TORCH_VERSION", TORCH_VERSION) < 0) Py_CLEAR(m);
  return m;
}

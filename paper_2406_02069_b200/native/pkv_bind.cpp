// Native half of the Python binding: checks the tensors of a call and hands it to the C boundary
// (include/pyramidkv.h) without going through ctypes.
//
// A per-layer call on a short context takes the GPU some 20 us, and one decode step makes a call per layer, so what the
// host spends per call is what such programs wait for.  Checks through tensor attributes and ctypes marshalling took 25
// of the 32 us that the host needed for a compress_layer call and 6.5 of the 9.3 us of a decode_attention call; with
// this file those calls take 7 and 2.8 us, launches included.
//
// Every function returns the C status (PKV_OK = 0, an error code otherwise), or kNotTaken when an argument is not what
// the quick checks accept: another kind of object, memory that is not on a CUDA device, a tensor that is too small.
// Nothing has been enqueued then; the caller goes through binding.py's own checks, which accept the rarer forms
// (pinned host memory) and raise the error with its reason for the rest.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <algorithm>
#include <cstring>
#include <vector>

#include <ATen/core/Tensor.h>
#include <c10/cuda/CUDAFunctions.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include "pyramidkv.h"

namespace {

constexpr int kNotTaken = -1;
PyObject* g_config_type = nullptr;       // PkvConfig: other objects that expose a buffer of its size are not configurations

// A tensor argument as the checks need it (borrowed: the arguments outlive the call).
struct View {
  const at::Tensor* t = nullptr;
  explicit operator bool() const { return t != nullptr; }
  void* ptr() const { return t->data_ptr(); }
  int64_t size(int i) const { return t->sizes()[i]; }
  int64_t stride(int i) const { return t->strides()[i]; }
  pkv_tensor strided() const { return pkv_tensor{t->data_ptr(), stride(0), stride(1), stride(2)}; }
};

bool get(PyObject* o, View* v) {
  if (!THPVariable_Check(o)) return false;
  const at::Tensor& t = THPVariable_Unpack(o);
  if (!t.defined() || t.layout() != c10::kStrided || !t.is_cuda() || !t.has_storage()) return false;
  v->t = &t;
  return true;
}

c10::ScalarType scalar_type(const pkv_config* c) {
  return c->dtype == PKV_DTYPE_FP32 ? c10::kFloat : (c->dtype == PKV_DTYPE_BF16 ? c10::kBFloat16 : c10::kHalf);
}

// What every call starts with: the configuration, the lengths and the stream.
struct Call {
  Py_buffer buf{};
  const pkv_config* cfg = nullptr;
  int32_t lens[PKV_MAX_BATCH];
  int32_t batch = 0;
  int32_t longest = 0;
  void* stream = nullptr;

  ~Call() { if (cfg) PyBuffer_Release(&buf); }

  bool open(PyObject* config, PyObject* seq_lens) {
    if (!g_config_type || PyObject_IsInstance(config, g_config_type) != 1) { PyErr_Clear(); return false; }
    if (PyObject_GetBuffer(config, &buf, PyBUF_SIMPLE) != 0) { PyErr_Clear(); return false; }
    cfg = static_cast<const pkv_config*>(buf.buf);               // released by the destructor from here on
    if (buf.len != static_cast<Py_ssize_t>(sizeof(pkv_config))) return false;
    if (cfg->num_kv_heads < 1 || cfg->dtype < PKV_DTYPE_FP32 || cfg->dtype > PKV_DTYPE_FP16) return false;
    const bool list = PyList_Check(seq_lens);
    if (!list && !PyTuple_Check(seq_lens)) return false;
    const Py_ssize_t n = list ? PyList_GET_SIZE(seq_lens) : PyTuple_GET_SIZE(seq_lens);
    if (n < 1 || n > PKV_MAX_BATCH) return false;
    for (Py_ssize_t i = 0; i < n; ++i) {
      PyObject* o = list ? PyList_GET_ITEM(seq_lens, i) : PyTuple_GET_ITEM(seq_lens, i);
      if (!PyLong_CheckExact(o)) return false;
      const long v = PyLong_AsLong(o);
      if ((v == -1 && PyErr_Occurred()) || v < cfg->window + 1l || v > INT32_MAX) { PyErr_Clear(); return false; }
      lens[i] = static_cast<int32_t>(v);
      longest = std::max(longest, lens[i]);
    }
    batch = static_cast<int32_t>(n);
    return true;
  }

  // Last of the checks: the current stream is only asked for once the tensors are known to live on a device.
  bool on_stream(PyObject* stream_or_none) {
    if (stream_or_none == Py_None) {
      stream = c10::cuda::getCurrentCUDAStream().stream();
    } else {
      PyObject* s = PyObject_GetAttrString(stream_or_none, "cuda_stream");
      if (!s) { PyErr_Clear(); return false; }
      stream = PyLong_AsVoidPtr(s);
      Py_DECREF(s);
      if (PyErr_Occurred()) { PyErr_Clear(); return false; }
    }
    return true;
  }

  // A K or V tensor as large as the call will read.
  bool kv(PyObject* o, View* v) const {
    return get(o, v) && v->t->dim() == 4 && v->stride(3) == 1 && v->t->scalar_type() == scalar_type(cfg) && v->size(0) >= batch &&
           v->size(1) == cfg->num_kv_heads && v->size(3) == cfg->head_dim && v->size(2) >= longest &&
           (batch == 1 || v->stride(0) > 0) && (cfg->num_kv_heads == 1 || v->stride(1) > 0) && v->stride(2) >= cfg->head_dim;
  }
  bool q(PyObject* o, View* v) const {
    return get(o, v) && v->t->dim() == 4 && v->stride(3) == 1 && v->t->scalar_type() == scalar_type(cfg) && v->size(0) >= batch &&
           v->size(1) == cfg->num_q_heads && v->size(2) == cfg->window && v->size(3) == cfg->head_dim;
  }
  bool scores(PyObject* o, View* v) const {
    const int64_t columns = longest - cfg->window;
    return get(o, v) && v->t->dim() == 3 && v->t->scalar_type() == c10::kFloat && v->size(0) >= batch &&
           v->size(1) == cfg->num_kv_heads && v->size(2) >= columns && v->stride(2) == 1 && v->stride(1) >= columns &&
           (batch == 1 || v->stride(0) == cfg->num_kv_heads * v->stride(1));
  }
  // A contiguous tensor of a type with at least so many elements.
  static bool flat(PyObject* o, View* v, c10::ScalarType type, int64_t least) {
    return get(o, v) && v->t->scalar_type() == type && v->t->is_contiguous() && v->t->numel() >= least;
  }
  bool lse(PyObject* o, View* v) const {
    return flat(o, v, c10::kFloat, static_cast<int64_t>(batch) * cfg->num_q_heads * cfg->window);
  }
  bool rows_out(PyObject* k, PyObject* v, PyObject* idx, int64_t rows, View* kv_, View* vv, View* iv) const {
    return flat(k, kv_, scalar_type(cfg), rows * cfg->head_dim) && flat(v, vv, scalar_type(cfg), rows * cfg->head_dim) &&
           flat(idx, iv, c10::kInt, rows);
  }
  static bool workspace(PyObject* o, View* v) { return flat(o, v, c10::kByte, 1); }
  bool attn_out(PyObject* o, View* v) const {
    return flat(o, v, c10::kFloat, 0) && v->t->dim() == 4 && v->size(0) == batch && v->size(1) == cfg->num_q_heads &&
           v->size(2) == cfg->window && v->size(3) == cfg->head_dim;
  }
  // Packed rows of a layer with budget k_layer, or a negative number for a configuration the library refuses.
  int64_t packed_rows(int32_t k_layer) const {
    int64_t rows = 0;
    for (int b = 0; b < batch; ++b) {
      const int c = pyramidkv_kept_count(cfg, k_layer, lens[b]);
      if (c < 0) return -1;
      rows += c;
    }
    return rows * cfg->num_kv_heads;
  }
  // ... of layer `layer`; the schedule of the last configuration is remembered per thread.
  int64_t layer_rows(int64_t layer) const {
    thread_local pkv_config last{};
    thread_local std::vector<int32_t> budgets;
    if (layer < 0 || layer >= cfg->num_layers) return -1;
    if (budgets.empty() || std::memcmp(&last, cfg, sizeof last) != 0) {
      budgets.assign(static_cast<size_t>(cfg->num_layers), 0);
      if (pyramidkv_layer_budgets(cfg, budgets.data()) != PKV_OK) { budgets.clear(); return -1; }
      last = *cfg;
    }
    return packed_rows(budgets[static_cast<size_t>(layer)]);
  }
};

bool as_int32(PyObject* o, int32_t* out) {
  if (!PyLong_Check(o)) return false;
  const long v = PyLong_AsLong(o);
  if (v < INT32_MIN || v > INT32_MAX || (v == -1 && PyErr_Occurred())) { PyErr_Clear(); return false; }
  *out = static_cast<int32_t>(v);
  return true;
}

PyObject* status(int rc) { return PyLong_FromLong(rc); }
PyObject* not_taken() { return PyLong_FromLong(kNotTaken); }

// Runs the C call with the interpreter's lock released, as ctypes does; the lock is taken again also when it throws.
template <typename F>
PyObject* without_gil(F&& f) {
  struct Release {
    PyThreadState* state = PyEval_SaveThread();
    ~Release() { PyEval_RestoreThread(state); }
  };
  int rc;
  {
    Release unlocked;
    rc = f();
  }
  return status(rc);
}

// (cfg, layer, q_win, k, v, seq_lens, k_out, v_out, indices, workspace, scores, stream, window_lse)
PyObject* compress_layer(PyObject*, PyObject* const* a, Py_ssize_t n) {
  Call c;
  View q, k, v, ko, vo, idx, ws, sc, lse;
  int32_t layer;
  if (n != 13 || !as_int32(a[1], &layer) || !c.open(a[0], a[5])) return not_taken();
  const int64_t rows = c.layer_rows(layer);
  if (rows < 0 || !c.q(a[2], &q) || !c.kv(a[3], &k) || !c.kv(a[4], &v) || !c.rows_out(a[6], a[7], a[8], rows, &ko, &vo, &idx) ||
      !Call::workspace(a[9], &ws) || (a[10] != Py_None && !c.scores(a[10], &sc)) || (a[12] != Py_None && !c.lse(a[12], &lse)) ||
      !c.on_stream(a[11]))
    return not_taken();
  float* s = sc ? static_cast<float*>(sc.ptr()) : nullptr;
  const int64_t ld = sc ? sc.stride(1) : 0;
  return without_gil([&] {
    return lse ? pyramidkv_compress_layer_lse(c.cfg, layer, q.strided(), k.strided(), v.strided(), static_cast<const float*>(lse.ptr()),
                                              c.lens, c.batch, ko.ptr(), vo.ptr(), static_cast<int32_t*>(idx.ptr()), s, ld, ws.ptr(),
                                              static_cast<size_t>(ws.t->numel()), c.stream)
               : pyramidkv_compress_layer(c.cfg, layer, q.strided(), k.strided(), v.strided(), c.lens, c.batch, ko.ptr(), vo.ptr(),
                                          static_cast<int32_t*>(idx.ptr()), s, ld, ws.ptr(), static_cast<size_t>(ws.t->numel()),
                                          c.stream);
  });
}

// (cfg, layer, q_win, k, v, seq_lens, attn_out, k_out, v_out, indices, workspace, scores, stream)
PyObject* attend_compress_layer(PyObject*, PyObject* const* a, Py_ssize_t n) {
  Call c;
  View q, k, v, at, ko, vo, idx, ws, sc;
  int32_t layer;
  if (n != 13 || !as_int32(a[1], &layer) || !c.open(a[0], a[5])) return not_taken();
  const int64_t rows = c.layer_rows(layer);
  if (rows < 0 || !c.q(a[2], &q) || !c.kv(a[3], &k) || !c.kv(a[4], &v) || !c.attn_out(a[6], &at) ||
      !c.rows_out(a[7], a[8], a[9], rows, &ko, &vo, &idx) || !Call::workspace(a[10], &ws) ||
      (a[11] != Py_None && !c.scores(a[11], &sc)) || !c.on_stream(a[12]))
    return not_taken();
  return without_gil([&] {
    return pyramidkv_attend_compress_layer(c.cfg, layer, q.strided(), k.strided(), v.strided(), c.lens, c.batch,
                                           static_cast<float*>(at.ptr()), ko.ptr(), vo.ptr(), static_cast<int32_t*>(idx.ptr()),
                                           sc ? static_cast<float*>(sc.ptr()) : nullptr, sc ? sc.stride(1) : 0, ws.ptr(),
                                           static_cast<size_t>(ws.t->numel()), c.stream);
  });
}

// Block table and pools of a paged call: [num_pages][page_size][d] pools of one shape.
bool paged(const Call& c, PyObject* table, PyObject* k, PyObject* v, View* tab, View* kp, View* vp) {
  return Call::flat(table, tab, c10::kInt, 0) && Call::flat(k, kp, scalar_type(c.cfg), 1) && Call::flat(v, vp, scalar_type(c.cfg), 1) &&
         kp->t->dim() == 3 && kp->t->sizes() == vp->t->sizes() && kp->size(2) == c.cfg->head_dim && kp->size(0) <= INT32_MAX &&
         kp->size(1) <= INT32_MAX;
}

// (cfg, layer, q_win, k, v, seq_lens, block_table, k_pool, v_pool, indices, workspace, scores, stream, window_lse)
PyObject* compress_layer_paged(PyObject*, PyObject* const* a, Py_ssize_t n) {
  Call c;
  View q, k, v, tab, kp, vp, idx, ws, sc, lse;
  int32_t layer;
  if (n != 14 || !as_int32(a[1], &layer) || !c.open(a[0], a[5])) return not_taken();
  const int64_t rows = c.layer_rows(layer);
  if (rows < 0 || !c.q(a[2], &q) || !c.kv(a[3], &k) || !c.kv(a[4], &v) || !paged(c, a[6], a[7], a[8], &tab, &kp, &vp) ||
      !Call::flat(a[9], &idx, c10::kInt, rows) || !Call::workspace(a[10], &ws) || (a[11] != Py_None && !c.scores(a[11], &sc)) ||
      (a[13] != Py_None && !c.lse(a[13], &lse)) || !c.on_stream(a[12]))
    return not_taken();
  return without_gil([&] {
    return pyramidkv_compress_layer_paged(
        c.cfg, layer, q.strided(), k.strided(), v.strided(), lse ? static_cast<const float*>(lse.ptr()) : nullptr, c.lens, c.batch,
        static_cast<const int32_t*>(tab.ptr()), static_cast<int32_t>(kp.size(1)), static_cast<int32_t>(kp.size(0)), kp.ptr(), vp.ptr(),
        static_cast<int32_t*>(idx.ptr()), sc ? static_cast<float*>(sc.ptr()) : nullptr, sc ? sc.stride(1) : 0, ws.ptr(),
        static_cast<size_t>(ws.t->numel()), c.stream);
  });
}

// (cfg, q_win, k, seq_lens, scores, workspace, stream, window_lse)
PyObject* score_window(PyObject*, PyObject* const* a, Py_ssize_t n) {
  Call c;
  View q, k, sc, ws, lse;
  if (n != 8 || !c.open(a[0], a[3]) || !c.q(a[1], &q) || !c.kv(a[2], &k) || !c.scores(a[4], &sc) || !Call::workspace(a[5], &ws) ||
      (a[7] != Py_None && !c.lse(a[7], &lse)) || !c.on_stream(a[6]))
    return not_taken();
  float* s = static_cast<float*>(sc.ptr());
  return without_gil([&] {
    return lse ? pyramidkv_score_window_lse(c.cfg, q.strided(), k.strided(), static_cast<const float*>(lse.ptr()), c.lens, c.batch, s,
                                            sc.stride(1), ws.ptr(), static_cast<size_t>(ws.t->numel()), c.stream)
               : pyramidkv_score_window(c.cfg, q.strided(), k.strided(), c.lens, c.batch, s, sc.stride(1), ws.ptr(),
                                        static_cast<size_t>(ws.t->numel()), c.stream);
  });
}

// (cfg, scores, seq_lens, k_layer, indices, workspace, stream)
PyObject* select_topk(PyObject*, PyObject* const* a, Py_ssize_t n) {
  Call c;
  View sc, idx, ws;
  int32_t kl;
  if (n != 7 || !as_int32(a[3], &kl) || !c.open(a[0], a[2]) || !c.scores(a[1], &sc)) return not_taken();
  const int64_t rows = c.packed_rows(kl);
  if (rows < 0 || !Call::flat(a[4], &idx, c10::kInt, rows) || !Call::workspace(a[5], &ws) || !c.on_stream(a[6])) return not_taken();
  return without_gil([&] {
    return pyramidkv_select_topk(c.cfg, static_cast<const float*>(sc.ptr()), sc.stride(1), c.lens, c.batch, kl,
                                 static_cast<int32_t*>(idx.ptr()), ws.ptr(), static_cast<size_t>(ws.t->numel()), c.stream);
  });
}

// (cfg, k, v, indices, seq_lens, k_layer, k_out, v_out, stream)
PyObject* gather_compact(PyObject*, PyObject* const* a, Py_ssize_t n) {
  Call c;
  View k, v, idx, ko, vo;
  int32_t kl;
  if (n != 9 || !as_int32(a[5], &kl) || !c.open(a[0], a[4]) || !c.kv(a[1], &k) || !c.kv(a[2], &v)) return not_taken();
  const int64_t rows = c.packed_rows(kl);
  if (rows < 0 || !c.rows_out(a[6], a[7], a[3], rows, &ko, &vo, &idx) || !c.on_stream(a[8])) return not_taken();
  return without_gil([&] {
    return pyramidkv_gather_compact(c.cfg, k.strided(), v.strided(), static_cast<const int32_t*>(idx.ptr()), c.lens, c.batch, kl,
                                    ko.ptr(), vo.ptr(), c.stream);
  });
}

// (cfg, q, k_cache, v_cache, seq_lens, k_layer, out, stream)
PyObject* decode_attention(PyObject*, PyObject* const* a, Py_ssize_t n) {
  Call c;
  View q, k, v, out;
  int32_t kl;
  if (n != 8 || !as_int32(a[5], &kl) || !c.open(a[0], a[4])) return not_taken();
  const int64_t rows = c.packed_rows(kl), elems = static_cast<int64_t>(c.batch) * c.cfg->num_q_heads * c.cfg->head_dim;
  const c10::ScalarType type = scalar_type(c.cfg);
  if (rows < 0 || !Call::flat(a[1], &q, type, elems) || !Call::flat(a[2], &k, type, rows * c.cfg->head_dim) ||
      !Call::flat(a[3], &v, type, rows * c.cfg->head_dim) || !Call::flat(a[6], &out, c10::kFloat, elems) || !c.on_stream(a[7]))
    return not_taken();
  return without_gil([&] {
    return pyramidkv_decode_attention(c.cfg, q.ptr(), k.ptr(), v.ptr(), c.lens, c.batch, kl, static_cast<float*>(out.ptr()), c.stream);
  });
}

// (cfg, q, block_table, k_pool, v_pool, seq_lens, k_layer, out, workspace, stream)
PyObject* decode_attention_paged(PyObject*, PyObject* const* a, Py_ssize_t n) {
  Call c;
  View q, tab, kp, vp, out, ws;
  int32_t kl;
  if (n != 10 || !as_int32(a[6], &kl) || !c.open(a[0], a[5])) return not_taken();
  const int64_t elems = static_cast<int64_t>(c.batch) * c.cfg->num_q_heads * c.cfg->head_dim;
  if (!Call::flat(a[1], &q, scalar_type(c.cfg), elems) || !paged(c, a[2], a[3], a[4], &tab, &kp, &vp) ||
      !Call::flat(a[7], &out, c10::kFloat, elems) || !Call::workspace(a[8], &ws) || !c.on_stream(a[9]))
    return not_taken();
  return without_gil([&] {
    return pyramidkv_decode_attention_paged(c.cfg, q.ptr(), kp.ptr(), vp.ptr(), static_cast<const int32_t*>(tab.ptr()),
                                            static_cast<int32_t>(kp.size(1)), static_cast<int32_t>(kp.size(0)), c.lens, c.batch, kl,
                                            static_cast<float*>(out.ptr()), ws.ptr(), static_cast<size_t>(ws.t->numel()), c.stream);
  });
}

// ---------------------------------------------------------------- growing cache
PyObject* g_cache_type = nullptr;        // cache.PkvCache, cache.PkvRotary
PyObject* g_rotary_type = nullptr;

// cache.PkvCache: the struct that the library takes, and behind it what it was made for.
struct CacheObject {
  pkv_cache cache;
  int32_t heads_kv, head_dim, dtype, device;
};

// A ctypes structure of a known type, read through its buffer.
struct Struct {
  Py_buffer buf{};
  ~Struct() { if (buf.obj) PyBuffer_Release(&buf); }
  const void* open(PyObject* o, PyObject* type, size_t size) {
    if (!type || PyObject_IsInstance(o, type) != 1 || PyObject_GetBuffer(o, &buf, PyBUF_SIMPLE) != 0) { PyErr_Clear(); return nullptr; }
    return buf.len == static_cast<Py_ssize_t>(size) ? buf.buf : nullptr;
  }
};

// What every call on a cache starts with.  A call without one (rotary) has the device of its tensors instead.
struct CacheCall {
  Struct cfg_buf, cache_buf, plan_buf;
  const pkv_config* cfg = nullptr;
  const CacheObject* of = nullptr;
  const pkv_rotary* plan = nullptr;
  int device = -1;
  void* stream = nullptr;

  bool open_config(PyObject* o) {
    cfg = static_cast<const pkv_config*>(cfg_buf.open(o, g_config_type, sizeof(pkv_config)));
    if (!cfg || cfg->num_kv_heads < 1 || cfg->dtype < PKV_DTYPE_FP32 || cfg->dtype > PKV_DTYPE_FP16) return false;
    device = c10::cuda::current_device();
    return true;
  }
  bool open_cache(PyObject* o, Struct* at, const CacheObject** out) const {
    *out = static_cast<const CacheObject*>(at->open(o, g_cache_type, sizeof(CacheObject)));
    return *out && (*out)->heads_kv == cfg->num_kv_heads && (*out)->head_dim == cfg->head_dim && (*out)->dtype == cfg->dtype && (*out)->device == device;
  }
  bool open(PyObject* config, PyObject* cache) { return open_config(config) && open_cache(cache, &cache_buf, &of); }
  bool open_plan(PyObject* o) {
    plan = static_cast<const pkv_rotary*>(plan_buf.open(o, g_rotary_type, sizeof(pkv_rotary)));
    return plan != nullptr;
  }
  bool on_stream(PyObject* stream_or_none) {
    if (stream_or_none == Py_None) {
      stream = c10::cuda::getCurrentCUDAStream().stream();
      return true;
    }
    PyObject* s = PyObject_GetAttrString(stream_or_none, "cuda_stream");
    if (!s) { PyErr_Clear(); return false; }
    stream = PyLong_AsVoidPtr(s);
    Py_DECREF(s);
    if (PyErr_Occurred()) { PyErr_Clear(); return false; }
    return true;
  }
  bool here(PyObject* o, View* v) const { return get(o, v) && v->t->get_device() == device; }
  // [batch][heads][tokens][d] rows of the configured type
  bool rows(PyObject* o, View* v, int64_t batch, int64_t heads, int64_t tokens) const {
    return here(o, v) && v->t->dim() == 4 && v->t->scalar_type() == scalar_type(cfg) && v->size(0) == batch && v->size(1) == heads &&
           v->size(2) == tokens && v->size(3) == cfg->head_dim && v->stride(3) == 1;
  }
  // A dimension of one entry has no say in where rows lie.
  pkv_tensor strided(const View& v) const {
    if (!v) return pkv_tensor{nullptr, 0, 0, 0};
    const int64_t d = cfg->head_dim;
    return pkv_tensor{v.ptr(), v.size(0) > 1 ? v.stride(0) : d, v.size(1) > 1 ? v.stride(1) : d, v.size(2) > 1 ? v.stride(2) : d};
  }
  bool positions(PyObject* o, View* v, int64_t batch, int64_t tokens, int64_t* stride) const {
    if (!here(o, v) || v->t->dim() != 2 || v->t->scalar_type() != c10::kInt || v->size(0) != batch || v->size(1) != tokens ||
        (tokens > 1 && v->stride(1) != 1))
      return false;
    *stride = batch > 1 ? v->stride(0) : 0;
    return true;
  }
  // A contiguous tensor of a type and shape (-1: dimension not there).
  bool shaped(PyObject* o, View* v, c10::ScalarType type, int64_t n0, int64_t n1 = -1, int64_t n2 = -1) const {
    const int dims = n1 < 0 ? 1 : (n2 < 0 ? 2 : 3);
    return here(o, v) && v->t->dim() == dims && v->t->scalar_type() == type && v->size(0) == n0 && (n1 < 0 || v->size(1) == n1) &&
           (n2 < 0 || v->size(2) == n2) && v->t->is_contiguous();
  }
  bool workspace(PyObject* o, View* v) const { return here(o, v) && v->t->scalar_type() == c10::kByte && v->t->is_contiguous(); }
  bool add(PyObject* o, View* v, int64_t batch, int64_t* stride) const {
    if (!here(o, v) || v->t->scalar_type() != c10::kInt) return false;
    const int64_t layers = of->cache.layers, last = v->t->dim() - 1;
    if (last == 0 ? v->size(0) != batch : (last != 1 || v->size(0) != layers || v->size(1) != batch)) return false;
    if (batch > 1 && v->stride(static_cast<int>(last)) != 1) return false;
    *stride = last == 1 && layers > 1 ? v->stride(0) : 0;
    return true;
  }
};

bool as_float(PyObject* o, float* out) {
  const double v = PyFloat_Check(o) ? PyFloat_AS_DOUBLE(o) : (PyLong_Check(o) ? PyLong_AsDouble(o) : -1.0);
  if (PyErr_Occurred()) { PyErr_Clear(); return false; }
  *out = static_cast<float>(v);
  return PyFloat_Check(o) || PyLong_Check(o);
}
int32_t* ints(const View& v) { return v ? static_cast<int32_t*>(v.ptr()) : nullptr; }
float* floats(const View& v) { return v ? static_cast<float*>(v.ptr()) : nullptr; }
size_t bytes_of(const View& ws) { return static_cast<size_t>(ws.t->numel()); }

// (cfg, plan, positions, q, k, q_out, k_out, inverse, stream); q or k and its output may be None
PyObject* rotary(PyObject*, PyObject* const* a, Py_ssize_t n) {
  CacheCall c;
  View pos, q, k, qo, ko;
  int64_t stride;
  if (n != 9 || !c.open_config(a[0]) || !c.open_plan(a[1])) return not_taken();
  PyObject* some = a[3] != Py_None ? a[3] : a[4];
  View first;
  if (!c.here(some, &first) || first.t->dim() != 4) return not_taken();
  const int64_t batch = first.size(0), tokens = first.size(2);
  if (batch < 1 || tokens < 1 || batch * tokens > INT32_MAX || !c.positions(a[2], &pos, batch, tokens, &stride)) return not_taken();
  if (a[3] != Py_None && (!c.rows(a[3], &q, batch, c.cfg->num_q_heads, tokens) || !c.rows(a[5], &qo, batch, c.cfg->num_q_heads, tokens))) return not_taken();
  if (a[4] != Py_None && (!c.rows(a[4], &k, batch, c.cfg->num_kv_heads, tokens) || !c.rows(a[6], &ko, batch, c.cfg->num_kv_heads, tokens))) return not_taken();
  if (!c.on_stream(a[8])) return not_taken();
  const int inverse = PyObject_IsTrue(a[7]);
  if (inverse < 0) { PyErr_Clear(); return not_taken(); }
  return without_gil([&] {
    return pyramidkv_rotary(c.cfg, c.plan, ints(pos), stride, static_cast<int32_t>(batch), static_cast<int32_t>(tokens), c.strided(q), c.strided(qo),
                            c.strided(k), c.strided(ko), inverse, c.stream);
  });
}

// (cfg, cache, layer, positions, k, v, workspace, q, q_out, plan, counts, stream)
PyObject* append_cache(PyObject*, PyObject* const* a, Py_ssize_t n) {
  CacheCall c;
  View pos, q, qo, k, v, counts, ws;
  int32_t layer;
  int64_t stride = 0;
  if (n != 12 || !as_int32(a[2], &layer) || !c.open(a[0], a[1]) || !c.here(a[4], &k) || k.t->dim() != 4) return not_taken();
  const int64_t batch = c.of->cache.batch, tokens = k.size(2);
  if (tokens < 1 || tokens > INT32_MAX || !c.rows(a[4], &k, batch, c.cfg->num_kv_heads, tokens) || !c.rows(a[5], &v, batch, c.cfg->num_kv_heads, tokens) ||
      !c.workspace(a[6], &ws) || (a[9] != Py_None && !c.open_plan(a[9])) ||
      (a[3] == Py_None ? c.plan || c.of->cache.positions : !c.positions(a[3], &pos, batch, tokens, &stride)) ||
      (a[10] != Py_None && !c.shaped(a[10], &counts, c10::kInt, batch)))
    return not_taken();
  if (a[7] != Py_None && (!c.rows(a[7], &q, batch, c.cfg->num_q_heads, tokens) || !c.rows(a[8], &qo, batch, c.cfg->num_q_heads, tokens))) return not_taken();
  if (!c.on_stream(a[11])) return not_taken();
  return without_gil([&] {
    return pyramidkv_append_cache(c.cfg, &c.of->cache, layer, c.plan, ints(pos), stride, static_cast<int32_t>(tokens), c.strided(q), c.strided(qo),
                                  c.strided(k), c.strided(v), ints(counts), ws.ptr(), bytes_of(ws), c.stream);
  });
}

// (cfg, cache, layer, q, out, workspace, q_positions, lse, scale, softcap, slopes, window, prefix, stream)
PyObject* decode_attention_cache(PyObject*, PyObject* const* a, Py_ssize_t n) {
  CacheCall c;
  View q, out, ws, pos, lse, slopes;
  int32_t layer;
  pkv_attend_options o{};
  if (n != 14 || !as_int32(a[2], &layer) || !c.open(a[0], a[1]) || !as_float(a[8], &o.scale) || !as_float(a[9], &o.softcap) ||
      !as_int32(a[11], &o.window) || !as_int32(a[12], &o.prefix))
    return not_taken();
  const int64_t batch = c.of->cache.batch, heads = c.cfg->num_q_heads, d = c.cfg->head_dim;
  if (!c.here(a[3], &q) || q.t->scalar_type() != scalar_type(c.cfg)) return not_taken();
  const int last = static_cast<int>(q.t->dim()) - 1;              // [batch][H_q][d] or [batch][H_q][1][d]
  if ((last != 2 && (last != 3 || q.size(2) != 1)) || q.size(0) != batch || q.size(1) != heads || q.size(last) != d || q.stride(last) != 1 ||
      !c.shaped(a[4], &out, c10::kFloat, batch, heads, d) || !c.workspace(a[5], &ws) || (a[6] != Py_None && !c.shaped(a[6], &pos, c10::kInt, batch)) ||
      (a[7] != Py_None && !c.shaped(a[7], &lse, c10::kFloat, batch, heads)) || (a[10] != Py_None && !c.shaped(a[10], &slopes, c10::kFloat, heads)) ||
      !c.on_stream(a[13]))
    return not_taken();
  o.slopes = floats(slopes);
  o.q_positions = ints(pos);
  const pkv_tensor view{q.ptr(), batch > 1 ? q.stride(0) : 0, heads > 1 ? q.stride(1) : 0, 0};
  return without_gil([&] {
    return pyramidkv_decode_attention_cache(c.cfg, &c.of->cache, layer, &o, view, floats(out), floats(lse), ws.ptr(), bytes_of(ws), c.stream);
  });
}

// (cfg, cache, to, add, granted, workspace, stream)
PyObject* cache_reserve(PyObject*, PyObject* const* a, Py_ssize_t n) {
  CacheCall c;
  Struct to_buf;
  const CacheObject* to;
  View add, granted, ws;
  int64_t stride;
  if (n != 7 || !c.open(a[0], a[1]) || !c.open_cache(a[2], &to_buf, &to) || !c.of->cache.refs || !to->cache.refs ||
      !c.add(a[3], &add, c.of->cache.batch, &stride) || (a[4] != Py_None && !c.shaped(a[4], &granted, c10::kInt, c.of->cache.layers, to->cache.batch)) ||
      !c.workspace(a[5], &ws) || !c.on_stream(a[6]))
    return not_taken();
  return without_gil([&] {
    return pyramidkv_cache_reserve(c.cfg, &c.of->cache, &to->cache, ints(add), stride, ints(granted), ws.ptr(), bytes_of(ws), c.stream);
  });
}

// (cfg, cache, to, parents, add, granted, workspace, stream)
PyObject* cache_fork(PyObject*, PyObject* const* a, Py_ssize_t n) {
  CacheCall c;
  Struct to_buf;
  const CacheObject* to;
  View parents, add, granted, ws;
  int64_t stride = 0;
  if (n != 8 || !c.open(a[0], a[1]) || !c.open_cache(a[2], &to_buf, &to) || !c.of->cache.refs || !to->cache.refs ||
      !c.shaped(a[3], &parents, c10::kInt, to->cache.batch) || (a[4] != Py_None && !c.add(a[4], &add, to->cache.batch, &stride)) ||
      (a[5] != Py_None && !c.shaped(a[5], &granted, c10::kInt, c.of->cache.layers, to->cache.batch)) || !c.workspace(a[6], &ws) || !c.on_stream(a[7]))
    return not_taken();
  return without_gil([&] {
    return pyramidkv_cache_fork(c.cfg, &c.of->cache, &to->cache, ints(parents), ints(add), stride, ints(granted), ws.ptr(), bytes_of(ws), c.stream);
  });
}

// (cfg, cache, to, used, workspace, stream)
PyObject* cache_compact(PyObject*, PyObject* const* a, Py_ssize_t n) {
  CacheCall c;
  Struct to_buf;
  const CacheObject* to;
  View used, ws;
  if (n != 6 || !c.open(a[0], a[1]) || !c.open_cache(a[2], &to_buf, &to) || !c.of->cache.refs || !to->cache.refs ||
      (a[3] != Py_None && !c.shaped(a[3], &used, c10::kInt, 1)) || !c.workspace(a[4], &ws) || !c.on_stream(a[5]))
    return not_taken();
  return without_gil([&] { return pyramidkv_cache_compact(c.cfg, &c.of->cache, &to->cache, ints(used), ws.ptr(), bytes_of(ws), c.stream); });
}

// A tensor that cannot be asked for its data (a fake one, say) or a CUDA runtime that does not answer throws: left to the
// other path too.
template <PyObject* (*F)(PyObject*, PyObject* const*, Py_ssize_t)>
PyObject* guarded(PyObject* self, PyObject* const* a, Py_ssize_t n) {
  try {
    return F(self, a, n);
  } catch (...) {
    PyErr_Clear();
    return not_taken();
  }
}

// (type): the class of the configurations.
PyObject* set_config_type(PyObject*, PyObject* type) {
  Py_INCREF(type);
  Py_XDECREF(g_config_type);
  g_config_type = type;
  Py_RETURN_NONE;
}

// (cache type, plan type): the classes of the growing cache's structures.
PyObject* set_cache_types(PyObject*, PyObject* const* a, Py_ssize_t n) {
  if (n != 2) { PyErr_SetString(PyExc_TypeError, "set_cache_types takes two classes"); return nullptr; }
  PyObject** to[2] = {&g_cache_type, &g_rotary_type};
  for (int i = 0; i < 2; ++i) {
    Py_INCREF(a[i]);
    Py_XDECREF(*to[i]);
    *to[i] = a[i];
  }
  Py_RETURN_NONE;
}

#define PKV_METHOD(name) {#name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)(void)>(guarded<name>)), METH_FASTCALL, nullptr}
PyMethodDef methods[] = {PKV_METHOD(compress_layer), PKV_METHOD(attend_compress_layer), PKV_METHOD(compress_layer_paged),
                         PKV_METHOD(score_window), PKV_METHOD(select_topk), PKV_METHOD(gather_compact), PKV_METHOD(decode_attention),
                         PKV_METHOD(decode_attention_paged), PKV_METHOD(rotary), PKV_METHOD(append_cache), PKV_METHOD(decode_attention_cache),
                         PKV_METHOD(cache_reserve), PKV_METHOD(cache_fork), PKV_METHOD(cache_compact),
                         {"set_cache_types", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)(void)>(set_cache_types)), METH_FASTCALL, nullptr},
                         {"set_config_type", set_config_type, METH_O, nullptr}, {nullptr, nullptr, 0, nullptr}};
PyModuleDef module_def = {PyModuleDef_HEAD_INIT, "_pkv_native", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__pkv_native() { return PyModule_Create(&module_def); }

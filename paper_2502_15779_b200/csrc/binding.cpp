// Argument marshalling of the calls a decode step makes once per layer, in native code: type, device, layout and shape
// checks of the tensors, their pointers, the current stream, the call. Marshalled by ctypes these calls cost the host 11
// to 13 us each, 6.6 of them outside the library (a Python stream object, an argument object per pointer), more than the
// GPU needs for a small layer. No computation here; the library's entry points are handed over by address
// (bind), so that the same module serves whichever build of it is loaded.
#include <Python.h>

#include <algorithm>
#include <climits>

#include <ATen/core/Tensor.h>
#include <c10/cuda/CUDAGuard.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include "../../include/rcp.h"

#ifndef RCP_HEADER_ID
#define RCP_HEADER_ID 0ull
#endif

namespace {

struct Entry {
  decltype(&rcp_quantize_act) quantize_act = nullptr;
  decltype(&rcp_gemv_w2a4_variant) gemv = nullptr;
  decltype(&rcp_gemv_w2a4_grouped_variant) gemv_grouped = nullptr;
  decltype(&rcp_gemv_w2a16_checked) gemv_w2a16 = nullptr;
  decltype(&rcp_gemv_w3a4) gemv_w3a4 = nullptr;
  decltype(&rcp_linear_w2a4_checked) linear = nullptr;
  decltype(&rcp_linear_w2a4_host) linear_host = nullptr;
  decltype(&rcp_gemv_workspace_bytes) workspace_bytes = nullptr;
  decltype(&rcp_kv_append) kv_append = nullptr;
  decltype(&rcp_kv_attention_variant) kv_attention = nullptr;
  decltype(&rcp_kv_attention_workspace_bytes) kv_workspace_bytes = nullptr;
  decltype(&rcp_lora_add) lora_add = nullptr;
  decltype(&rcp_lora_workspace_bytes) lora_workspace_bytes = nullptr;
} g_fn;


const char* type_name(at::ScalarType t) {
  return t == at::kHalf ? "float16" : t == at::kInt ? "int32" : t == at::kFloat ? "float32" : t == at::kChar ? "int8" : t == at::kFloat8_e4m3fn ? "float8_e4m3fn" : "uint8";
}
bool on_other_device(const char* name) {
  PyErr_Format(PyExc_ValueError, "%s: not on the device of the call's first tensor", name);
  return false;
}
// A contiguous CUDA tensor of the given type (on the device of `like`), or a TypeError.
const at::Tensor* dev(PyObject* o, at::ScalarType type, const char* name, const at::Tensor* like = nullptr) {
  if (THPVariable_Check(o)) {
    const at::Tensor& t = THPVariable_Unpack(o);
    if (t.is_cuda() && t.scalar_type() == type && t.is_contiguous()) {
      if (like && t.device() != like->device()) { on_other_device(name); return nullptr; }
      return &t;
    }
  }
  PyErr_Format(PyExc_TypeError, "%s: expected a contiguous CUDA tensor of dtype torch.%s", name, type_name(type));
  return nullptr;
}
// The address of an optional buffer (None: null) that the library knows nothing else of: at least `need` elements of the given
// type (kByte: or int8; kAny: bytes of any type), contiguous, on the device of `like` or in page-locked host memory, which
// the device reaches as well.
constexpr at::ScalarType kAny = at::ScalarType::Undefined;
bool buffer(PyObject* o, const char* name, at::ScalarType type, const at::Tensor& like, int64_t need, void** out) {
  *out = nullptr;
  if (o == Py_None) return true;
  if (!THPVariable_Check(o)) {
    PyErr_Format(PyExc_TypeError, "%s: expected a tensor or None", name);
    return false;
  }
  const at::Tensor& t = THPVariable_Unpack(o);
  const at::ScalarType have = t.scalar_type();
  if (have == type && t.is_cuda() && t.numel() >= need && t.is_contiguous() && t.get_device() == like.get_device()) {   // as a rule
    *out = t.data_ptr();
    return true;
  }
  const bool fits = type == kAny || have == type || ((type == at::kByte || type == at::kChar) && (have == at::kByte || have == at::kChar));
  if (!fits || !t.is_contiguous() || !(t.is_cuda() || t.is_pinned())) {
    PyErr_Format(PyExc_TypeError, "%s: expected a contiguous CUDA tensor%s%s", name, type == kAny ? "" : " of dtype torch.",
                 type == kAny ? "" : type_name(type));
    return false;
  }
  if (t.is_cuda() && t.device() != like.device()) return on_other_device(name);
  if ((type == kAny ? (int64_t)t.nbytes() : t.numel()) < need) {
    PyErr_Format(PyExc_ValueError, "%s: %lld %s, %lld are needed", name, (long long)(type == kAny ? (int64_t)t.nbytes() : t.numel()),
                 type == kAny ? "bytes" : "elements", (long long)need);
    return false;
  }
  *out = t.data_ptr();
  return true;
}
// bytes of workspace the library wants (0 for shapes it refuses)
int64_t workspace_bytes(int64_t M, int64_t N, int64_t K) { return (int64_t)g_fn.workspace_bytes((int)M, (int)N, (int)K); }
bool has_shape(const at::Tensor& t, std::initializer_list<int64_t> want) { return t.sizes() == at::IntArrayRef(want); }
bool bad_shapes(const char* what) {
  PyErr_Format(PyExc_ValueError, "shape mismatch between %s", what);
  return false;
}
// What int(o) and float(o) take: whole-numbered floats, numpy scalars, one-element tensors as well.
bool integer(PyObject* o, int* out) {
  long x;
  if (PyLong_CheckExact(o)) {
    x = PyLong_AsLong(o);
  } else {
    PyObject* v = PyNumber_Long(o);
    if (!v) return false;
    x = PyLong_AsLong(v);
    Py_DECREF(v);
  }
  if (x == -1 && PyErr_Occurred()) return false;
  *out = (int)x;
  return true;
}
bool real(PyObject* o, float* out) {
  if (PyFloat_CheckExact(o)) {
    *out = (float)PyFloat_AS_DOUBLE(o);
    return true;
  }
  PyObject* v = PyNumber_Float(o);
  if (!v) return false;
  const double x = PyFloat_AS_DOUBLE(v);
  Py_DECREF(v);
  *out = (float)x;
  return true;
}
// What a call returns to Python: its status (0: done).
PyObject* status(int rc) { return PyLong_FromLong(rc); }

// Runs `call(stream)` with t's device current and its current stream, without the interpreter lock.
template <typename Call>
PyObject* on_device(const at::Tensor& t, Call call) {
  int rc;
  const c10::cuda::CUDAGuard guard(t.device());
  void* const stream = c10::cuda::getCurrentCUDAStream(t.device().index()).stream();
  Py_BEGIN_ALLOW_THREADS
  rc = call(stream);
  Py_END_ALLOW_THREADS
  return status(rc);
}
bool count(Py_ssize_t have, Py_ssize_t want) {
  if (have == want) return true;
  PyErr_Format(PyExc_TypeError, "expected %zd arguments, got %zd", want, have);
  return false;
}

// C++ exceptions of the tensor library become RuntimeErrors
template <typename F>
PyObject* guarded(F f) {
  try {
    return f();
  } catch (const std::exception& e) {
    PyErr_SetString(PyExc_RuntimeError, e.what());
    return nullptr;
  }
}

// bind({name: address}): the loaded library's entry points
PyObject* bind(PyObject*, PyObject* table) {
  if (!PyDict_Check(table)) {
    PyErr_SetString(PyExc_TypeError, "bind: a dict of addresses is expected");
    return nullptr;
  }
  auto take = [&](const char* name, auto& fn) {
    PyObject* v = PyDict_GetItemString(table, name);   // borrowed
    if (!v) {
      PyErr_Format(PyExc_KeyError, "bind: %s is missing", name);
      return false;
    }
    void* const p = PyLong_AsVoidPtr(v);
    if (PyErr_Occurred()) return false;
    fn = reinterpret_cast<std::decay_t<decltype(fn)>>(p);
    return true;
  };
  if (!take("rcp_quantize_act", g_fn.quantize_act) || !take("rcp_gemv_w2a4_variant", g_fn.gemv) ||
      !take("rcp_gemv_w2a4_grouped_variant", g_fn.gemv_grouped) || !take("rcp_gemv_w2a16_checked", g_fn.gemv_w2a16) ||
      !take("rcp_gemv_w3a4", g_fn.gemv_w3a4) || !take("rcp_linear_w2a4_checked", g_fn.linear) ||
      !take("rcp_linear_w2a4_host", g_fn.linear_host) || !take("rcp_gemv_workspace_bytes", g_fn.workspace_bytes) ||
      !take("rcp_kv_append", g_fn.kv_append) || !take("rcp_kv_attention_variant", g_fn.kv_attention) ||
      !take("rcp_kv_attention_workspace_bytes", g_fn.kv_workspace_bytes) || !take("rcp_lora_add", g_fn.lora_add) ||
      !take("rcp_lora_workspace_bytes", g_fn.lora_workspace_bytes))
    return nullptr;
  decltype(&rcp_header_id) header_id = nullptr;
  if (!take("rcp_header_id", header_id)) return nullptr;
  if (header_id() != RCP_HEADER_ID) {
    g_fn = {};
    PyErr_SetString(PyExc_RuntimeError, "the library and its marshalling module were not built from the same include/rcp.h: build both anew "
                                        "with `python -m paper_2502_15779_b200.build`");
    return nullptr;
  }
  Py_RETURN_NONE;
}

// (x, had_block, clip_ratio, xq, scale)
PyObject* quantize_act(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded([&]() -> PyObject* {
    int B;
    float clip;
    void *xq, *scale;
    if (!count(n, 5)) return nullptr;
    const at::Tensor* x = dev(a[0], at::kHalf, "x");
    if (!x || !integer(a[1], &B) || !real(a[2], &clip)) return nullptr;
    if (x->dim() != 2) { bad_shapes("x and [M][K]"); return nullptr; }
    const int M = (int)x->size(0), K = (int)x->size(1);
    if (!buffer(a[3], "xq", at::kByte, *x, x->size(0) * (x->size(1) / 2), &xq) || !buffer(a[4], "scale", at::kHalf, *x, x->size(0), &scale))
      return nullptr;
    const void* const xp = x->data_ptr();
    return on_device(*x, [&](void* st) { return g_fn.quantize_act(xp, M, K, B, clip, static_cast<uint8_t*>(xq), scale, st); });
  });
}

// (variant, words, lut, group, xq, scale, y, workspace, S_dbg); group 0: one grid per row
PyObject* gemv_w2a4(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded([&]() -> PyObject* {
    int variant, group;
    void *y, *ws, *S;
    if (!count(n, 9) || !integer(a[0], &variant) || !integer(a[3], &group)) return nullptr;
    const at::Tensor* words = dev(a[1], at::kInt, "words");
    if (!words) return nullptr;
    const at::Tensor* lut = dev(a[2], at::kHalf, "lut", words);
    if (!lut) return nullptr;
    const at::Tensor* xq = dev(a[4], at::kByte, "xq", words);
    if (!xq) return nullptr;
    const at::Tensor* scale = dev(a[5], at::kHalf, "scale", words);
    if (!scale) return nullptr;
    const bool two = words->dim() == 2 && xq->dim() == 2;
    const int64_t N = two ? words->size(0) : 0, K = two ? 16 * words->size(1) : 0, M = two ? xq->size(0) : 0;
    const bool grid = group == 0 ? has_shape(*lut, {N, 4}) : group > 0 && K % group == 0 && has_shape(*lut, {N, K / group, 4});
    if (!two || !grid || !has_shape(*xq, {M, K / 2}) || !has_shape(*scale, {M})) {
      bad_shapes(group == 0 ? "words, lut, xq and scale" : "words, lut, group, xq and scale");
      return nullptr;
    }
    if (!buffer(a[6], "y", at::kHalf, *words, M * N, &y) || !buffer(a[7], "workspace", kAny, *words, workspace_bytes(M, N, K), &ws) ||
        !buffer(a[8], "S_dbg", at::kInt, *words, M * N * (group ? K / group : 1) * 4, &S))
      return nullptr;
    const uint32_t* const wp = static_cast<const uint32_t*>(words->data_ptr());
    const void *lp = lut->data_ptr(), *sp = scale->data_ptr();
    const uint8_t* const qp = static_cast<const uint8_t*>(xq->data_ptr());
    return on_device(*words, [&](void* st) {
      return group == 0 ? g_fn.gemv(variant, wp, lp, qp, sp, (int)M, (int)N, (int)K, y, ws, static_cast<int32_t*>(S), st)
                        : g_fn.gemv_grouped(variant, wp, lp, group, qp, sp, (int)M, (int)N, (int)K, y, ws, static_cast<int32_t*>(S), st);
    });
  });
}

// (words, lut, x, y, digits, unit, workspace, S_dbg)
PyObject* gemv_w2a16(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded([&]() -> PyObject* {
    void *y, *digits, *unit, *ws, *S;
    if (!count(n, 8)) return nullptr;
    const at::Tensor* words = dev(a[0], at::kInt, "words");
    if (!words) return nullptr;
    const at::Tensor* lut = dev(a[1], at::kHalf, "lut", words);
    if (!lut) return nullptr;
    const at::Tensor* x = dev(a[2], at::kHalf, "x", words);
    if (!x) return nullptr;
    const bool two = words->dim() == 2 && x->dim() == 2;
    const int64_t N = two ? words->size(0) : 0, K = two ? 16 * words->size(1) : 0, M = two ? x->size(0) : 0;
    if (!two || !has_shape(*x, {M, K}) || !has_shape(*lut, {N, 4})) { bad_shapes("words, lut and x"); return nullptr; }
    if (!buffer(a[3], "y", at::kHalf, *words, M * N, &y) || !buffer(a[4], "digits", at::kChar, *words, M * 4 * K, &digits) ||
        !buffer(a[5], "unit", at::kFloat, *words, M * 4, &unit) ||
        !buffer(a[6], "workspace", kAny, *words, workspace_bytes(M, N, K), &ws) || !buffer(a[7], "S_dbg", at::kInt, *words, 4 * M * N * 4, &S))
      return nullptr;
    const uint32_t* const wp = static_cast<const uint32_t*>(words->data_ptr());
    const void *lp = lut->data_ptr(), *xp = x->data_ptr();
    return on_device(*words, [&](void* st) {
      return g_fn.gemv_w2a16(wp, lp, xp, (int)M, (int)N, (int)K, y, static_cast<int8_t*>(digits), static_cast<float*>(unit), ws,
                             static_cast<int32_t*>(S), st);
    });
  });
}

// (words2, words1, lut, group, xq, scale, y, S_dbg)
PyObject* gemv_w3a4(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded([&]() -> PyObject* {
    int group;
    void *y, *S;
    if (!count(n, 8) || !integer(a[3], &group)) return nullptr;
    const at::Tensor* words2 = dev(a[0], at::kInt, "words2");
    if (!words2) return nullptr;
    const at::Tensor* words1 = dev(a[1], at::kInt, "words1", words2);
    if (!words1) return nullptr;
    const at::Tensor* lut = dev(a[2], at::kHalf, "lut", words2);
    if (!lut) return nullptr;
    const at::Tensor* xq = dev(a[4], at::kByte, "xq", words2);
    if (!xq) return nullptr;
    const at::Tensor* scale = dev(a[5], at::kHalf, "scale", words2);
    if (!scale) return nullptr;
    const bool two = words2->dim() == 2 && xq->dim() == 2;
    const int64_t N = two ? words2->size(0) : 0, K = two ? 16 * words2->size(1) : 0, M = two ? xq->size(0) : 0;
    const bool grid = group == 0 ? has_shape(*lut, {N, 8}) : has_shape(*lut, {N, K / std::max(group, 1), 8});
    if (!two || !grid || !has_shape(*words1, {N, K / 32}) || !has_shape(*xq, {M, K / 2}) || !has_shape(*scale, {M})) {
      bad_shapes("words2, words1, lut, group, xq and scale");
      return nullptr;
    }
    if (!buffer(a[6], "y", at::kHalf, *words2, M * N, &y) ||
        !buffer(a[7], "S_dbg", at::kInt, *words2, M * N * (group ? K / std::max(group, 1) : 1) * 8, &S))
      return nullptr;
    const uint32_t *w2 = static_cast<const uint32_t*>(words2->data_ptr()), *w1 = static_cast<const uint32_t*>(words1->data_ptr());
    const void *lp = lut->data_ptr(), *sp = scale->data_ptr();
    const uint8_t* const qp = static_cast<const uint8_t*>(xq->data_ptr());
    return on_device(*words2, [&](void* st) {
      return g_fn.gemv_w3a4(w2, w1, lp, group, qp, sp, (int)M, (int)N, (int)K, y, static_cast<int32_t*>(S), st);
    });
  });
}

// (x, had_block, clip_ratio, words, lut, group, y, xq, scale, workspace, S_dbg)
PyObject* linear_w2a4(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded([&]() -> PyObject* {
    int B, group;
    float clip;
    void *y, *xq, *scale, *ws, *S;
    if (!count(n, 11)) return nullptr;
    const at::Tensor* x = dev(a[0], at::kHalf, "x");
    if (!x) return nullptr;
    const at::Tensor* words = dev(a[3], at::kInt, "words", x);
    if (!words) return nullptr;
    const at::Tensor* lut = dev(a[4], at::kHalf, "lut", x);
    if (!lut || !integer(a[1], &B) || !real(a[2], &clip) || !integer(a[5], &group)) return nullptr;
    const bool two = words->dim() == 2 && x->dim() == 2;
    const int64_t N = two ? words->size(0) : 0, K = two ? x->size(1) : 0, M = two ? x->size(0) : 0;
    const bool grid = group == 0 ? has_shape(*lut, {N, 4}) : has_shape(*lut, {N, K / std::max(group, 1), 4});
    if (!two || words->size(1) * 16 != K || !grid) { bad_shapes("x, words, lut and group"); return nullptr; }
    if (!buffer(a[6], "y", at::kHalf, *x, M * N, &y) || !buffer(a[7], "xq", at::kByte, *x, M * (K / 2), &xq) ||
        !buffer(a[8], "scale", at::kHalf, *x, M, &scale) || !buffer(a[9], "workspace", kAny, *x, workspace_bytes(M, N, K), &ws) ||
        !buffer(a[10], "S_dbg", at::kInt, *x, M * N * (group ? K / std::max(group, 1) : 1) * 4, &S))
      return nullptr;
    const uint32_t* const wp = static_cast<const uint32_t*>(words->data_ptr());
    const void *lp = lut->data_ptr(), *xp = x->data_ptr();
    return on_device(*words, [&](void* st) {
      return g_fn.linear(xp, (int)M, (int)K, B, clip, wp, lp, group, (int)N, y, static_cast<uint8_t*>(xq), scale, ws,
                         static_cast<int32_t*>(S), st);
    });
  });
}

// (x_host, had_block, clip_ratio, words, lut, y_host, x_dev, xq_dev, scale_dev, y_dev, workspace)
PyObject* linear_w2a4_host(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded([&]() -> PyObject* {
    int B;
    float clip;
    void *xd, *xq, *scale, *yd, *ws;
    if (!count(n, 11)) return nullptr;
    if (!THPVariable_Check(a[0]) || !THPVariable_Check(a[5])) {
      PyErr_SetString(PyExc_TypeError, "x_host and y_host must be tensors");
      return nullptr;
    }
    const at::Tensor &x = THPVariable_Unpack(a[0]), &y = THPVariable_Unpack(a[5]);
    if (!x.is_cpu() || !y.is_cpu() || x.scalar_type() != at::kHalf || y.scalar_type() != at::kHalf || !x.is_contiguous() ||
        !y.is_contiguous()) {
      PyErr_SetString(PyExc_TypeError, "x_host / y_host must be contiguous fp16 host tensors");
      return nullptr;
    }
    const at::Tensor* words = dev(a[3], at::kInt, "words");
    if (!words) return nullptr;
    const at::Tensor* lut = dev(a[4], at::kHalf, "lut", words);
    if (!lut || !integer(a[1], &B) || !real(a[2], &clip)) return nullptr;
    const bool two = words->dim() == 2 && x.dim() == 2;
    const int64_t N = two ? words->size(0) : 0, K = two ? x.size(1) : 0, M = two ? x.size(0) : 0;
    if (!two || words->size(1) * 16 != K || lut->numel() != 4 * N || y.numel() < M * N) {
      bad_shapes("x_host, words, lut and y_host");
      return nullptr;
    }
    if (!buffer(a[6], "x_dev", at::kHalf, *words, M * K, &xd) || !buffer(a[7], "xq_dev", at::kByte, *words, M * (K / 2), &xq) ||
        !buffer(a[8], "scale_dev", at::kHalf, *words, M, &scale) || !buffer(a[9], "y_dev", at::kHalf, *words, M * N, &yd) ||
        !buffer(a[10], "workspace", kAny, *words, workspace_bytes(M, N, K), &ws))
      return nullptr;
    const void *const xp = x.data_ptr(), *const lp = lut->data_ptr();
    void* const yp = y.data_ptr();
    const uint32_t* const wp = static_cast<const uint32_t*>(words->data_ptr());
    return on_device(*words, [&](void* st) {
      return g_fn.linear_host(xp, (int)M, (int)K, B, clip, wp, lp, (int)N, yp, xd, static_cast<uint8_t*>(xq), scale, yd, ws, st);
    });
  });
}

// fp16 rows of `dims` - 1 packed dimensions, the rows any distance apart (parts of a fused projection): a TypeError otherwise
const at::Tensor* rows(PyObject* o, const char* name, int dims, const at::Tensor* like, int64_t* stride) {
  if (THPVariable_Check(o)) {
    const at::Tensor& t = THPVariable_Unpack(o);
    if (t.is_cuda() && t.scalar_type() == at::kHalf && t.dim() == dims) {
      bool packed = t.size(dims - 1) == 1 || t.stride(dims - 1) == 1;
      if (dims == 3) packed = packed && (t.size(1) == 1 || t.stride(1) == t.size(2));
      if (packed) {
        if (like && t.device() != like->device()) { on_other_device(name); return nullptr; }
        *stride = t.size(0) == 1 ? (dims == 3 ? t.size(1) * t.size(2) : t.size(1)) : t.stride(0);
        return &t;
      }
    }
  }
  PyErr_Format(PyExc_TypeError, "%s: expected a CUDA tensor of dtype torch.float16 with %d dimensions, all but the first without gaps", name, dims);
  return nullptr;
}
// The paged cache and the sequences, as both calls on it take them: a[0..3] k, v, k_scale, v_scale; a[4..6] starts, lengths, table
struct Cache {
  const at::Tensor *k, *v, *ks, *vs, *starts, *lengths, *table;
  int pages, kv_heads, page, dim, seqs, width;
};
bool cache_of(PyObject* const* a, const at::Tensor* like, Cache* c) {
  if (!(c->k = dev(a[0], at::kFloat8_e4m3fn, "cache.k", like)) || !(c->v = dev(a[1], at::kFloat8_e4m3fn, "cache.v", like)) ||
      !(c->ks = dev(a[2], at::kFloat, "cache.k_scale", like)) || !(c->vs = dev(a[3], at::kFloat, "cache.v_scale", like)) ||
      !(c->starts = dev(a[4], at::kInt, "starts", like)) || !(c->lengths = dev(a[5], at::kInt, "lengths", like)) ||
      !(c->table = dev(a[6], at::kInt, "block_table", like)))
    return false;
  const at::Tensor &k = *c->k, &t = *c->table;
  if (k.dim() != 4 || k.sizes() != c->v->sizes() || !has_shape(*c->ks, {k.size(0), k.size(1)}) || c->ks->sizes() != c->vs->sizes())
    return bad_shapes("the cache's codes [pages][kv_heads][page][dim] and scales [pages][kv_heads]");
  if (t.dim() != 2 || !has_shape(*c->lengths, {t.size(0)}) || !has_shape(*c->starts, {t.size(0) + 1}))
    return bad_shapes("starts [seqs + 1], lengths [seqs] and block_table [seqs][width]");
  for (int64_t n : {k.size(0), k.size(1), k.size(2), k.size(3), t.size(0), t.size(1)})
    if (n > INT_MAX) return bad_shapes("the cache and its table: a size beyond 31 bits");
  c->pages = (int)k.size(0); c->kv_heads = (int)k.size(1); c->page = (int)k.size(2); c->dim = (int)k.size(3);
  c->seqs = (int)t.size(0); c->width = (int)t.size(1);
  return true;
}
const int32_t* ints(const at::Tensor* t) { return static_cast<const int32_t*>(t->data_ptr()); }

// (k, v, cache.k, cache.v, cache.k_scale, cache.v_scale, starts, lengths, block_table, rope, interleaved, q, q_out, max_new)
PyObject* kv_append(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded([&]() -> PyObject* {
    Cache c;
    int64_t ks, vs, qs = 0;
    int interleaved, max_new;
    void* q_out = nullptr;
    if (!count(n, 14)) return nullptr;
    const at::Tensor* k = rows(a[0], "k", 3, nullptr, &ks);
    if (!k) return nullptr;
    const at::Tensor* v = rows(a[1], "v", 3, k, &vs);
    if (!v || !cache_of(a + 2, k, &c) || !integer(a[10], &interleaved) || !integer(a[13], &max_new)) return nullptr;
    const int64_t T = k->size(0);
    if (T > INT_MAX || !has_shape(*k, {T, c.kv_heads, c.dim}) || v->sizes() != k->sizes()) { bad_shapes("k, v and the cache"); return nullptr; }
    const at::Tensor *rope = nullptr, *q = nullptr;
    if (a[9] != Py_None) {
      if (!(rope = dev(a[9], at::kFloat, "rope", k))) return nullptr;
      if (rope->dim() != 3 || rope->size(2) != 2 || rope->size(0) > INT_MAX || rope->size(1) > c.dim) {
        bad_shapes("rope and [positions][pairs][2]");
        return nullptr;
      }
    }
    int heads = c.kv_heads;
    if (a[11] != Py_None) {
      if (!(q = rows(a[11], "q", 3, k, &qs))) return nullptr;
      if (q->size(0) != T || q->size(2) != c.dim || q->size(1) > INT_MAX) { bad_shapes("q, k and v"); return nullptr; }
      heads = (int)q->size(1);
      if (!buffer(a[12], "q_out", at::kHalf, *k, q->numel(), &q_out)) return nullptr;
    }
    const void *kp = k->data_ptr(), *vp = v->data_ptr(), *qp = q ? q->data_ptr() : nullptr;
    const float* rp = rope ? static_cast<const float*>(rope->data_ptr()) : nullptr;
    void *kc = c.k->data_ptr(), *vc = c.v->data_ptr();
    float *ksc = static_cast<float*>(c.ks->data_ptr()), *vsc = static_cast<float*>(c.vs->data_ptr());
    const int32_t *st = ints(c.starts), *ln = ints(c.lengths), *tb = ints(c.table);
    if (T == 0) {   // empty tensors have no address; the library looks at none of these then
      kp = vp = kc;
      if (q) qp = q_out = kc;
    }
    const int positions = rope ? (int)rope->size(0) : 0, rot = rope ? 2 * (int)rope->size(1) : 0;
    return on_device(*k, [&](void* stream) {
      return g_fn.kv_append(qp, qs, kp, ks, vp, vs, (int)T, heads, c.kv_heads, c.dim, rp, positions, rot, interleaved, st, ln, tb, c.seqs, c.width,
                            max_new, kc, vc, ksc, vsc, c.pages, c.page, q_out, stream);
    });
  });
}

// (q, cache.k, cache.v, cache.k_scale, cache.v_scale, starts, lengths, block_table, sm_scale, max_new, out, workspace, variant)
PyObject* kv_attention(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded([&]() -> PyObject* {
    Cache c;
    int64_t qs;
    int max_new, variant;
    float sm_scale;
    void *out, *ws;
    if (!count(n, 13) || !integer(a[12], &variant)) return nullptr;
    const at::Tensor* q = rows(a[0], "q", 3, nullptr, &qs);
    if (!q || !cache_of(a + 1, q, &c) || !real(a[8], &sm_scale) || !integer(a[9], &max_new)) return nullptr;
    const int64_t T = q->size(0), heads = q->size(1);
    if (T > INT_MAX || heads > INT_MAX || q->size(2) != c.dim) { bad_shapes("q and the cache"); return nullptr; }
    if (!buffer(a[10], "out", at::kHalf, *q, q->numel(), &out) || !buffer(a[11], "workspace", kAny, *q, (int64_t)g_fn.kv_workspace_bytes(), &ws))
      return nullptr;
    const void *qp = q->data_ptr(), *kc = c.k->data_ptr(), *vc = c.v->data_ptr();
    if (T == 0) qp = out = c.k->data_ptr();   // as in kv_append
    const float *ksc = static_cast<const float*>(c.ks->data_ptr()), *vsc = static_cast<const float*>(c.vs->data_ptr());
    const int32_t *st = ints(c.starts), *ln = ints(c.lengths), *tb = ints(c.table);
    return on_device(*q, [&](void* stream) {
      return g_fn.kv_attention(variant, -1, qp, qs, (int)T, (int)heads, c.kv_heads, c.dim, sm_scale, st, ln, tb, c.seqs, c.width, max_new, kc, vc, ksc, vsc, c.pages,
                               c.page, out, ws, stream);
    });
  });
}

// (x, a, b, adapter, scaling, base, y, workspace)
PyObject* lora_add(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded([&]() -> PyObject* {
    int64_t xs;
    void *base, *y, *ws;
    if (!count(n, 8)) return nullptr;
    const at::Tensor* x = rows(a[0], "x", 2, nullptr, &xs);
    if (!x) return nullptr;
    const at::Tensor* down = dev(a[1], at::kHalf, "a", x);
    if (!down) return nullptr;
    const at::Tensor* up = dev(a[2], at::kHalf, "b", x);
    if (!up) return nullptr;
    const at::Tensor* adapter = dev(a[3], at::kInt, "adapter", x);
    if (!adapter) return nullptr;
    const at::Tensor* scaling = dev(a[4], at::kFloat, "scaling", x);
    if (!scaling) return nullptr;
    const int64_t M = x->size(0), K = x->size(1);
    if (down->dim() != 3 || up->dim() != 3) { bad_shapes("x, a, b, adapter and scaling"); return nullptr; }
    const int64_t L = down->size(0), R = down->size(1), N = up->size(1);
    if (!has_shape(*down, {L, R, K}) || !has_shape(*up, {L, N, R}) || !has_shape(*adapter, {M}) || !has_shape(*scaling, {L}) || M > INT_MAX ||
        N > INT_MAX || K > INT_MAX || L > INT_MAX) {
      bad_shapes("x, a, b, adapter and scaling");
      return nullptr;
    }
    if (!buffer(a[5], "base", at::kHalf, *x, M * N, &base) || !buffer(a[6], "y", at::kHalf, *x, M * N, &y) ||
        !buffer(a[7], "workspace", kAny, *x, (int64_t)g_fn.lora_workspace_bytes((int)M, (int)std::min<int64_t>(R, INT_MAX)), &ws))
      return nullptr;
    const void *xp = x->data_ptr(), *ap = down->data_ptr(), *bp = up->data_ptr();
    const int32_t* ip = ints(adapter);
    const float* sp = static_cast<const float*>(scaling->data_ptr());
    return on_device(*x, [&](void* st) {
      return g_fn.lora_add(xp, xs, ap, bp, ip, sp, base, (int)M, (int)N, (int)K, (int)R, (int)L, y, ws, st);
    });
  });
}

#define RCP_FAST(fn) {#fn, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(fn)), METH_FASTCALL, nullptr}
PyMethodDef kMethods[] = {{"bind", bind, METH_O, nullptr}, RCP_FAST(quantize_act), RCP_FAST(gemv_w2a4), RCP_FAST(gemv_w2a16),
                          RCP_FAST(gemv_w3a4), RCP_FAST(linear_w2a4), RCP_FAST(linear_w2a4_host),
                          RCP_FAST(kv_append), RCP_FAST(kv_attention), RCP_FAST(lora_add), {nullptr, nullptr, 0, nullptr}};
PyModuleDef kModule = {PyModuleDef_HEAD_INIT, "_marshal", nullptr, -1, kMethods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__marshal() { return PyModule_Create(&kModule); }

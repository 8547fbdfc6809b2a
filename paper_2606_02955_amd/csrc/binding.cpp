// binding.cpp -- the attention calls on torch tensors: each checks its tensors,
// takes their addresses and strides and calls libfdllm.so.  They are made once
// a layer on a few tokens at a time, where a launch takes 2 to 3 us and checking
// and converting two dozen arguments in Python took 6 more.
#include <torch/csrc/autograd/python_variable.h>

#include <ATen/ops/empty.h>

#include <cmath>
#include <cstdint>
#include <exception>
#include <initializer_list>
#include <stdexcept>
#include <string>

#include "fdllm.h"

namespace {

typedef std::initializer_list<int64_t> Shape;

std::string text(const int64_t* d, size_t n) {
  std::string s = "(";
  for (size_t i = 0; i < n; ++i) s += (i ? ", " : "") + std::to_string(d[i]);
  return s + (n == 1 ? ",)" : ")");
}

const at::Tensor& tensor(PyObject* o, const char* name) {
  if (!THPVariable_Check(o)) throw std::invalid_argument(std::string(name) + " must be a tensor");
  return THPVariable_Unpack(o);
}

// A tensor on the GPU of a type and shape.
void expect(const at::Tensor& t, at::ScalarType type, Shape shape, const char* name) {
  if (!t.is_cuda()) throw std::invalid_argument(std::string(name) + " must be a GPU tensor");
  if (t.scalar_type() != type)
    throw std::invalid_argument(std::string(name) + " must be " + c10::toString(type) + ", got " + c10::toString(t.scalar_type()));
  const auto s = t.sizes();
  if (s.size() != shape.size() || !std::equal(s.begin(), s.end(), shape.begin()))
    throw std::invalid_argument(std::string(name) + " must have shape " + text(shape.begin(), shape.size()) + ", got " +
                                text(s.data(), s.size()));
}

// Address of a contiguous one.
void* at_of(PyObject* o, at::ScalarType type, Shape shape, const char* name) {
  const at::Tensor& t = tensor(o, name);
  expect(t, type, shape, name);
  if (!t.is_contiguous()) throw std::invalid_argument(std::string(name) + " must be contiguous");
  return t.data_ptr();
}
void* at_or_null(PyObject* o, at::ScalarType type, Shape shape, const char* name) {
  return o == Py_None ? nullptr : at_of(o, type, shape, name);
}

// [T, heads, D] whose tokens may lie apart: address and elements from token to token.
struct Heads {
  void* p = nullptr;
  int64_t stride = 0;
};
Heads heads_of(PyObject* o, at::ScalarType type, int64_t T, int64_t H, int64_t D, const char* name) {
  const at::Tensor& t = tensor(o, name);
  expect(t, type, {T, H, D}, name);
  if ((t.stride(1) != D && H != 1) || (t.stride(2) != 1 && D != 1))
    throw std::invalid_argument(std::string(name) + ": the heads of a token must lie side by side");
  return {t.data_ptr(), T > 1 ? t.stride(0) : H * D};
}

const at::Tensor& dims(PyObject* o, int64_t n, const char* name, const char* what) {
  const at::Tensor& t = tensor(o, name);
  if (t.dim() != n) {
    const auto s = t.sizes();
    throw std::invalid_argument(std::string(name) + " must be " + what + ", got " + text(s.data(), s.size()));
  }
  return t;
}
const at::Tensor& rows(PyObject* o, const char* name) { return dims(o, 3, name, "[tokens, heads, head size]"); }

int whole(int64_t v, const char* name) {
  if (v < INT32_MIN || v > INT32_MAX) throw std::invalid_argument(std::string(name) + " does not fit 32 bits");
  return (int)v;
}
int whole(PyObject* o, const char* name) {
  const long long v = PyLong_AsLongLong(o);
  if (v == -1 && PyErr_Occurred()) {
    PyErr_Clear();
    throw std::invalid_argument(std::string(name) + " must be a whole number");
  }
  return whole((int64_t)v, name);
}
float real(PyObject* o, const char* name) {
  const double v = PyFloat_AsDouble(o);
  if (v == -1.0 && PyErr_Occurred()) {
    PyErr_Clear();
    throw std::invalid_argument(std::string(name) + " must be a number");
  }
  return (float)v;
}
bool truth(PyObject* o, const char* name) {
  const int v = PyObject_IsTrue(o);
  if (v < 0) {
    PyErr_Clear();
    throw std::invalid_argument(std::string(name) + " must be true or false");
  }
  return v != 0;
}
fdllm_stream stream_of(PyObject* o) { return (fdllm_stream)PyLong_AsVoidPtr(o); }

uint8_t* cache_of(PyObject* o, int64_t Hk, int64_t D, int* n_pages) {
  const at::Tensor& t = dims(o, 3, "cache", "[pages, key heads, tile bytes]");
  size_t tile = 0;
  if (fdllm_cache_tile_bytes(whole(D, "head size"), &tile) != FDLLM_OK)
    throw std::invalid_argument("no cache has heads of " + std::to_string(D) + " elements");
  *n_pages = whole(t.size(0), "cache pages");
  return (uint8_t*)at_of(o, at::kByte, {t.size(0), Hk, (int64_t)tile}, "cache");
}

// The caller's workspace, or a new one of the bytes needed (none: no tensor).
struct Scratch {
  at::Tensor own;
  void* p = nullptr;
  size_t bytes = 0;
};
Scratch scratch(PyObject* o, size_t need, const at::Tensor& like) {
  Scratch s;
  if (o != Py_None) {
    const at::Tensor& t = tensor(o, "workspace");
    if (!t.is_cuda() || !t.is_contiguous()) throw std::invalid_argument("workspace must be a contiguous GPU tensor");
    s.p = t.data_ptr();
    s.bytes = t.nbytes();
  } else if (need) {
    s.own = at::empty({(int64_t)need}, like.options().dtype(at::kByte));
    s.p = s.own.data_ptr();
    s.bytes = need;
  }
  return s;
}

// Status codes go back as whole numbers; what the tensors are wrong in, and
// anything that torch throws, as a Python error.
template <typename F>
PyObject* guarded(Py_ssize_t given, Py_ssize_t wanted, F&& f) {
  if (given != wanted) return PyErr_Format(PyExc_TypeError, "%zd arguments wanted, %zd given", wanted, given);
  try {
    return f();
  } catch (const std::invalid_argument& e) {
    PyErr_SetString(PyExc_ValueError, e.what());
  } catch (const std::bad_alloc&) {
    PyErr_NoMemory();
  } catch (const c10::Error& e) {
    PyErr_SetString(PyExc_RuntimeError, e.what_without_backtrace());
  } catch (const std::exception& e) {
    PyErr_SetString(PyExc_RuntimeError, e.what());
  }
  return nullptr;
}

template <typename F>
fdllm_status unlocked(F&& call) {
  fdllm_status st;
  Py_BEGIN_ALLOW_THREADS
  st = call();
  Py_END_ALLOW_THREADS
  return st;
}

PyObject* result(fdllm_status st, PyObject* given, const Scratch& s) {
  if (st != FDLLM_OK) return PyLong_FromLong(st);
  if (s.own.defined()) return THPVariable_Wrap(s.own);
  Py_INCREF(given);
  return given;
}

PyObject* qk_norm_rope(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded(n, 14, [&]() -> PyObject* {
    const at::Tensor& q = rows(a[0], "q");
    const int64_t T = q.size(0), H = q.size(1), D = q.size(2), Hk = rows(a[1], "k").size(1);
    const at::ScalarType type = q.scalar_type();
    if (type != at::kBFloat16 && type != at::kFloat) throw std::invalid_argument("q must be bfloat16 or float32");
    const Heads hq = heads_of(a[0], type, T, H, D, "q"), hk = heads_of(a[1], type, T, Hk, D, "k");
    Heads hv;
    uint8_t* cache = nullptr;
    const int32_t* slots = nullptr;
    int n_pages = 0;
    if (a[11] != Py_None) {
      if (a[2] == Py_None || a[12] == Py_None) throw std::invalid_argument("v and slots must be given with a cache");
      hv = heads_of(a[2], type, T, Hk, D, "v");
      cache = cache_of(a[11], Hk, D, &n_pages);
      slots = (const int32_t*)at_of(a[12], at::kInt, {T}, "slots");
    }
    int n_pos = 0, rot = 0;
    const float* table = nullptr;
    if (a[4] != Py_None) {
      const at::Tensor& t = dims(a[4], 2, "cos_sin", "[positions, rotated elements]");
      n_pos = whole(t.size(0), "cos_sin rows"), rot = whole(t.size(1), "cos_sin columns");
      table = (const float*)at_of(a[4], at::kFloat, {t.size(0), t.size(1)}, "cos_sin");
    }
    const float* qw = (const float*)at_or_null(a[7], at::kFloat, {D}, "q_weight");
    const float* kw = (const float*)at_or_null(a[8], at::kFloat, {D}, "k_weight");
    const int32_t* pos = (const int32_t*)at_of(a[3], at::kInt, {T}, "positions");
    void* q_out = at_of(a[5], type, {T, H, D}, "q_out");
    void* k_out = at_or_null(a[6], type, {T, Hk, D}, "k_out");
    const float eps = real(a[9], "eps");
    const int inter = truth(a[10], "interleaved"), t32 = whole(T, "tokens"), h32 = whole(H, "heads"),
              hk32 = whole(Hk, "heads"), d32 = whole(D, "head size");
    const fdllm_stream st = stream_of(a[13]);
    return PyLong_FromLong(unlocked([&] {
      return fdllm_qk_norm_rope(hq.p, hq.stride, hk.p, hk.stride, hv.p, hv.stride,
                                type == at::kFloat ? FDLLM_F32 : FDLLM_BF16, t32, h32, hk32, d32, qw, kw, eps, pos, table,
                                n_pos, rot, inter, q_out, k_out, cache, n_pages, slots, st);
    }));
  });
}

PyObject* cache_read(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded(n, 5, [&]() -> PyObject* {
    PyObject* like = a[2] != Py_None ? a[2] : a[3];
    if (like == Py_None) throw std::invalid_argument("k_out or v_out must be given");
    const at::Tensor& t = rows(like, "k_out");
    const int64_t T = t.size(0), Hk = t.size(1), D = t.size(2);
    const at::ScalarType type = t.scalar_type();
    if (type != at::kBFloat16 && type != at::kFloat8_e5m2)
      throw std::invalid_argument("the cache is read as bfloat16 or float8_e5m2");
    int n_pages = 0;
    const uint8_t* cache = cache_of(a[0], Hk, D, &n_pages);
    const int32_t* slots = (const int32_t*)at_of(a[1], at::kInt, {T}, "slots");
    void* k_out = at_or_null(a[2], type, {T, Hk, D}, "k_out");
    void* v_out = at_or_null(a[3], type, {T, Hk, D}, "v_out");
    const int t32 = whole(T, "tokens"), hk32 = whole(Hk, "heads"), d32 = whole(D, "head size");
    const fdllm_stream st = stream_of(a[4]);
    return PyLong_FromLong(unlocked([&] {
      return fdllm_cache_read(cache, n_pages, hk32, d32, slots, t32,
                              type == at::kBFloat16 ? FDLLM_OUT_BF16 : FDLLM_OUT_E5M2, k_out, v_out, st);
    }));
  });
}

// A number, or 1 / sqrt(head size) where none is given.
float scale_of(PyObject* o, int64_t D) { return o == Py_None ? (float)(1.0 / std::sqrt((double)D)) : real(o, "scale"); }

PyObject* cache_attention(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded(n, 13, [&]() -> PyObject* {
    const at::Tensor& q = rows(a[0], "q");
    const int64_t T = q.size(0), H = q.size(1), D = q.size(2);
    const Heads hq = heads_of(a[0], at::kBFloat16, T, H, D, "q");
    const int64_t Hk = dims(a[1], 3, "cache", "[pages, key heads, tile bytes]").size(1);
    int n_pages = 0;
    const uint8_t* cache = cache_of(a[1], Hk, D, &n_pages);
    const at::Tensor& table = dims(a[2], 2, "page_table", "[sequences, pages]");
    const int64_t B = table.size(0), width = table.size(1);
    const int32_t* tp = (const int32_t*)at_of(a[2], at::kInt, {B, width}, "page_table");
    const int32_t* kv = (const int32_t*)at_of(a[3], at::kInt, {B}, "kv_len");
    const int32_t* cu = (const int32_t*)at_of(a[4], at::kInt, {B + 1}, "cu_q");
    void* out = at_of(a[5], at::kBFloat16, {T, H, D}, "out");
    const int max_q = whole(a[6], "max_q"), blk = whole(a[9], "blk");
    float* lse = (float*)at_or_null(a[7], at::kFloat, {T, H}, "lse");
    const float scale = scale_of(a[8], D);
    const int32_t* start = (const int32_t*)at_or_null(a[10], at::kInt, {B}, "q_start");
    const int t32 = whole(T, "tokens"), b32 = whole(B, "sequences"), h32 = whole(H, "heads"), hk32 = whole(Hk, "heads"),
              d32 = whole(D, "head size"), w32 = whole(width, "page_table columns");
    size_t need = 0;
    if (a[11] == Py_None) {
      const fdllm_status st = fdllm_cache_attention_workspace_size(b32, h32, hk32, d32, max_q, w32, &need);
      if (st != FDLLM_OK) return PyLong_FromLong(st);
    }
    const Scratch ws = scratch(a[11], need, q);
    const fdllm_stream stream = stream_of(a[12]);
    return result(unlocked([&] {
      return fdllm_cache_attention(hq.p, hq.stride, t32, cu, b32, max_q, h32, hk32, d32, cache, n_pages, tp, w32, kv,
                                   start, scale, blk, out, lse, ws.p, ws.bytes, stream);
    }), a[11], ws);
  });
}

PyObject* prompt_attention(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded(n, 12, [&]() -> PyObject* {
    const at::Tensor& q = rows(a[0], "q");
    const at::Tensor& k = rows(a[1], "k");
    const int64_t T = q.size(0), H = q.size(1), D = q.size(2), Tk = k.size(0), Hk = k.size(1);
    const Heads hq = heads_of(a[0], at::kBFloat16, T, H, D, "q"), hk = heads_of(a[1], at::kBFloat16, Tk, Hk, D, "k"),
                hv = heads_of(a[2], at::kBFloat16, Tk, Hk, D, "v");
    const int64_t B = dims(a[3], 1, "cu_q", "[sequences + 1]").size(0) - 1;
    const int32_t* cu_q = (const int32_t*)at_of(a[3], at::kInt, {B + 1}, "cu_q");
    const int32_t* cu_k = (const int32_t*)at_of(a[4], at::kInt, {B + 1}, "cu_k");
    void* out = at_of(a[5], at::kBFloat16, {T, H, D}, "out");
    const int max_q = whole(a[6], "max_q"), blk = whole(a[9], "blk");
    float* lse = (float*)at_or_null(a[7], at::kFloat, {T, H}, "lse");
    const float scale = scale_of(a[8], D);
    const int t32 = whole(T, "tokens"), tk32 = whole(Tk, "keys"), b32 = whole(B, "sequences"), h32 = whole(H, "heads"),
              hk32 = whole(Hk, "heads"), d32 = whole(D, "head size");
    size_t need = 0;
    if (a[10] == Py_None) {
      const fdllm_status st = fdllm_prompt_attention_workspace_size(b32, t32, tk32, h32, hk32, d32, max_q, blk, &need);
      if (st != FDLLM_OK) return PyLong_FromLong(st);
    }
    const Scratch ws = scratch(a[10], need, q);
    const fdllm_stream stream = stream_of(a[11]);
    return result(unlocked([&] {
      return fdllm_prompt_attention(hq.p, hq.stride, hk.p, hk.stride, hv.p, hv.stride, t32, tk32, cu_q, cu_k, b32, max_q,
                                    h32, hk32, d32, scale, blk, out, lse, ws.p, ws.bytes, stream);
    }), a[10], ws);
  });
}

#define FDLLM_METHOD(f) {#f, (PyCFunction)(void (*)(void))f, METH_FASTCALL, nullptr}
PyMethodDef methods[] = {FDLLM_METHOD(qk_norm_rope), FDLLM_METHOD(cache_read), FDLLM_METHOD(cache_attention),
                         FDLLM_METHOD(prompt_attention), {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_binding", "The attention calls on torch tensors.", -1, methods,
                      nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__binding() { return PyModule_Create(&module); }

// The Python side of the calls of a decode step: tensors in, arguments of the C entry points out.
//
// A layer's step makes four of these calls on a few rows, where a call's time is the host's.  Looking at its ten tensors
// from Python takes longer than the launch (12.0 us a call of cs_qk_norm_rope through ctypes, 3.0 of them the launch), so
// these are looked at here.  Nothing is decided here: the checks are those that only the tensors allow (types, places, sizes
// that the C entry point cannot see), the rest is the entry point's.
//
// Every function takes its arguments by position, raises TypeError / ValueError for tensors that do not fit, and returns the status
// of the C call in place of its result where that is not CS_OK (binding.py has the signatures and raises CsError).
#include <Python.h>
#include <ATen/core/Tensor.h>
#include <ATen/ops/empty.h>
#include <c10/core/DeviceGuard.h>
#include <c10/hip/HIPStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include <cmath>
#include <exception>
#include <string>

#include "../../include/cornenc.h"

namespace {

struct Type : std::exception {
  std::string text;
  explicit Type(std::string t) : text(std::move(t)) {}
};
struct Value : std::exception {
  std::string text;
  explicit Value(std::string t) : text(std::move(t)) {}
};

const at::Tensor& tensor(PyObject* o, const char* name) {
  if (!THPVariable_Check(o)) throw Type(std::string(name) + ": expected a tensor");
  return THPVariable_Unpack(o);
}
int64_t number(PyObject* o) {
  const long long v = PyLong_AsLongLong(o);
  if (v == -1 && PyErr_Occurred()) throw Type("");        // (the error is set)
  return v;
}
int32_t number32(PyObject* o) {
  const int64_t v = number(o);
  if (v != (int32_t)v) throw Value("a size does not fit 32 bits");
  return (int32_t)v;
}
double real(PyObject* o) {
  const double v = PyFloat_AsDouble(o);
  if (v == -1.0 && PyErr_Occurred()) throw Type("");
  return v;
}
int32_t truth(PyObject* o) {
  const int v = PyObject_IsTrue(o);
  if (v < 0) throw Type("");
  return v;
}

int dtype_code(const at::Tensor& x) {
  if (x.scalar_type() == at::kBFloat16) return CS_BF16;
  if (x.scalar_type() == at::kFloat) return CS_F32;
  throw Type("rows must be bf16 or fp32");
}

// The device of a call is that of its first tensor
struct Call {
  c10::Device device;
  explicit Call(const at::Tensor& first, const char* name) : device(first.device()) {
    if (!first.is_cuda()) throw Value(std::string(name) + ": expected a tensor on the GPU");
  }
  void* stream() const { return c10::hip::getCurrentHIPStream(device.index()).stream(); }

  // [rows, heads, dim] with packed heads; rows may lie apart
  struct Rows {
    void* p;
    int64_t row;
  };
  Rows rows(const at::Tensor& x, int64_t heads, int64_t dim, const char* name) const {
    const auto s = x.strides();
    if (x.device() != device || s[2] != 1 || (s[1] != dim && heads > 1))
      throw Value(std::string(name) + ": heads of a row must be packed, on the GPU");
    return {x.data_ptr(), s[0] >= heads * dim || x.size(0) > 1 ? s[0] : heads * dim};
  }
  // the same of a tensor to be written, or one that has to be like another
  Rows given(const at::Tensor& x, int64_t n, int64_t heads, int64_t dim, at::ScalarType type, const char* name) const {
    if (x.dim() != 3 || x.size(0) != n || x.size(1) != heads || x.size(2) != dim || x.scalar_type() != type)
      throw Value(std::string(name) + ": expected [" + std::to_string(n) + ", " + std::to_string(heads) + ", " + std::to_string(dim) +
                  "] of the rows' type");
    return rows(x, heads, dim, name);
  }
  void* flat(const at::Tensor& x, at::ScalarType type, int64_t size, const char* name) const {
    if (x.scalar_type() != type || x.numel() != size || !x.is_contiguous() || x.device() != device)
      throw Value(std::string(name) + ": expected a contiguous tensor of " + std::to_string(size) + " elements of its type on the GPU");
    return x.data_ptr();
  }
  void* flat(PyObject* o, at::ScalarType type, int64_t size, const char* name) const { return flat(tensor(o, name), type, size, name); }
  void* optional(PyObject* o, at::ScalarType type, int64_t size, const char* name) const {
    return o == Py_None ? nullptr : flat(o, type, size, name);
  }
};

void three(const at::Tensor& x, const char* name) {
  if (x.dim() != 3) throw Value(std::string(name) + ": expected [rows, heads, head_dim]");
}

// the pool [n_pages, page bytes] of a cache
cs_cache_config cache_of(const Call& call, PyObject* o, int64_t kv_heads, int64_t dim, int64_t page_tokens, void*& p) {
  const at::Tensor& pool = tensor(o, "pool");
  if (pool.dim() != 2 || kv_heads > 1 << 20 || page_tokens > 1 << 30 || dim > 1 << 20 || pool.size(1) != kv_heads * page_tokens * (dim + dim / 16))
    throw Value("pool: expected [n_pages, page bytes] as cs_cache_query says");
  p = call.flat(pool, at::kByte, pool.numel(), "pool");
  return {sizeof(cs_cache_config), (int32_t)kv_heads, (int32_t)dim, (int32_t)page_tokens, pool.size(0)};
}

PyObject* status_or(int status, PyObject* result) {
  if (status == CS_OK) return result;
  Py_DECREF(result);
  return PyLong_FromLong(status);
}

template <class F>
PyObject* guarded(Py_ssize_t n, Py_ssize_t expected, F&& body) {
  if (n != expected) {
    PyErr_SetString(PyExc_TypeError, "wrong number of arguments");
    return nullptr;
  }
  try {
    return body();
  } catch (const Type& e) {
    if (!PyErr_Occurred()) PyErr_SetString(PyExc_TypeError, e.text.c_str());
  } catch (const Value& e) {
    PyErr_SetString(PyExc_ValueError, e.text.c_str());
  } catch (const c10::OutOfMemoryError& e) {
    PyObject *torch = PyImport_ImportModule("torch"), *type = torch ? PyObject_GetAttrString(torch, "OutOfMemoryError") : nullptr;
    PyErr_SetString(type ? type : PyExc_MemoryError, e.what_without_backtrace());
    Py_XDECREF(type);
    Py_XDECREF(torch);
  } catch (const std::exception& e) {
    PyErr_SetString(PyExc_RuntimeError, e.what());
  } catch (...) {
    PyErr_SetString(PyExc_RuntimeError, "unknown exception");
  }
  return nullptr;
}

// (q, k, cos_sin, positions, sections, q_gain, k_gain, eps, interleaved, q_out, k_out, err_flag) -> (q_out, k_out)
PyObject* qk_norm_rope(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded(n, 12, [&]() -> PyObject* {
    const at::Tensor &q = tensor(a[0], "q"), &k = tensor(a[1], "k"), &cs = tensor(a[2], "cos_sin");
    three(q, "q");
    three(k, "k");
    const Call call(q, "q");
    const int64_t T = q.size(0), H = q.size(1), D = q.size(2), K = k.size(1);
    if (cs.dim() != 3 || cs.size(2) != 2) throw Value("cos_sin: expected [n_positions, pairs, 2]");
    const int64_t axes = PySequence_Size(a[4]);
    if (axes < 0) throw Type("");
    if (axes > 3) throw Value("sections: at most three axes");
    if (H > 1 << 20 || K > 1 << 20 || D > 1 << 20 || cs.size(1) > 1 << 20) throw Value("q, k, cos_sin: sizes");
    const int code = dtype_code(q);
    cs_qk_config c = {sizeof(cs_qk_config), (int32_t)H, (int32_t)K, (int32_t)D, (int32_t)(2 * cs.size(1)), (int32_t)axes, truth(a[8]),
                      {0, 0, 0}, cs.size(0), (float)real(a[7])};
    for (int64_t i = 0; i < axes; ++i) {
      PyObject* item = PySequence_GetItem(a[4], i);
      if (!item) throw Type("");
      const long long v = PyLong_AsLongLong(item);
      Py_DECREF(item);
      if (v == -1 && PyErr_Occurred()) throw Type("");
      if (v != (int32_t)v) throw Value("sections: a size does not fit 32 bits");
      c.sections[i] = (int32_t)v;
    }
    const auto qr = call.rows(q, H, D, "q"), kr = call.given(k, T, K, D, q.scalar_type(), "k");
    void *qg = call.optional(a[5], at::kFloat, D, "q_gain"), *kg = call.optional(a[6], at::kFloat, D, "k_gain");
    void *table = call.flat(cs, at::kFloat, cs.numel(), "cos_sin"), *pos = call.flat(a[3], at::kInt, T * axes, "positions");
    void* flag = call.optional(a[11], at::kInt, 1, "err_flag");
    const at::Tensor qo = a[9] == Py_None ? at::empty({T, H, D}, q.options()) : tensor(a[9], "q_out");
    const at::Tensor ko = a[10] == Py_None ? at::empty({T, K, D}, q.options()) : tensor(a[10], "k_out");
    const auto qw = call.given(qo, T, H, D, q.scalar_type(), "q_out"), kw = call.given(ko, T, K, D, q.scalar_type(), "k_out");
    const int st = cs_qk_norm_rope(&c, qr.p, qr.row, kr.p, kr.row, qw.p, qw.row, kw.p, kw.row, code, static_cast<float*>(qg), static_cast<float*>(kg),
                                   static_cast<float*>(table), static_cast<int32_t*>(pos), T, static_cast<int32_t*>(flag), call.stream());
    if (st != CS_OK) return PyLong_FromLong(st);
    PyObject *x = THPVariable_Wrap(qo), *y = x ? THPVariable_Wrap(ko) : nullptr, *both = y ? PyTuple_Pack(2, x, y) : nullptr;
    Py_XDECREF(x);
    Py_XDECREF(y);
    return both;
  });
}

// (pool, k, v, slots, page_tokens, err_flag) -> None
PyObject* cache_write(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded(n, 6, [&]() -> PyObject* {
    const at::Tensor &k = tensor(a[1], "k"), &v = tensor(a[2], "v");
    three(k, "k");
    const Call call(k, "k");
    const int64_t T = k.size(0), K = k.size(1), D = k.size(2);
    const int code = dtype_code(k);
    void* pool;
    const cs_cache_config c = cache_of(call, a[0], K, D, number(a[4]), pool);
    const auto kr = call.rows(k, K, D, "k"), vr = call.given(v, T, K, D, k.scalar_type(), "v");
    const int st = cs_cache_write(&c, pool, kr.p, kr.row, vr.p, vr.row, code, static_cast<int64_t*>(call.flat(a[3], at::kLong, T, "slots")), T,
                                  static_cast<int32_t*>(call.optional(a[5], at::kInt, 1, "err_flag")), call.stream());
    Py_INCREF(Py_None);
    return status_or(st, Py_None);
  });
}

// (pool, slots, n_kv_heads, head_dim, page_tokens, dtype code, k, v, err_flag) -> (k, v)
PyObject* cache_read(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded(n, 9, [&]() -> PyObject* {
    const at::Tensor& slots = tensor(a[1], "slots");
    const Call call(slots, "slots");
    const int64_t T = slots.numel(), K = number32(a[2]), D = number32(a[3]);
    const int code = number32(a[5]);
    if (K <= 0 || D <= 0) throw Value("n_kv_heads, head_dim: expected sizes");
    void* pool;
    const cs_cache_config c = cache_of(call, a[0], K, D, number(a[4]), pool);
    const at::ScalarType type = code == CS_BF16 ? at::kBFloat16 : at::kFloat;
    const auto options = slots.options().dtype(type);
    void* at_slots = call.flat(slots, at::kLong, T, "slots");
    void* flag = call.optional(a[8], at::kInt, 1, "err_flag");
    const at::Tensor k = a[6] == Py_None ? at::empty({T, K, D}, options) : tensor(a[6], "k");
    const at::Tensor v = a[7] == Py_None ? at::empty({T, K, D}, options) : tensor(a[7], "v");
    const auto kr = call.given(k, T, K, D, type, "k"), vr = call.given(v, T, K, D, type, "v");
    const int st = cs_cache_read(&c, pool, static_cast<int64_t*>(at_slots), T, kr.p, kr.row, vr.p, vr.row, code, static_cast<int32_t*>(flag), call.stream());
    if (st != CS_OK) return PyLong_FromLong(st);
    PyObject *x = THPVariable_Wrap(k), *y = x ? THPVariable_Wrap(v) : nullptr, *both = y ? PyTuple_Pack(2, x, y) : nullptr;
    Py_XDECREF(x);
    Py_XDECREF(y);
    return both;
  });
}

// (q, pool, page_table, n_keys, cu_queries, max_queries, max_keys, n_kv_heads, page_tokens, scale, causal, out, workspace, err_flag) -> out
PyObject* attention_cache(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded(n, 14, [&]() -> PyObject* {
    const at::Tensor &q = tensor(a[0], "q"), &table = tensor(a[2], "page_table");
    three(q, "q");
    if (q.scalar_type() != at::kBFloat16) throw Type("q must be bf16");
    if (table.dim() != 2) throw Value("page_table: expected [sequences, pages]");
    const Call call(q, "q");
    const int64_t T = q.size(0), H = q.size(1), D = q.size(2), B = table.size(0), width = table.size(1);
    if (H > 1 << 20 || B > 0x7fffffff || width > 0x7fffffff) throw Value("q, page_table: sizes");
    void* pool;
    const cs_cache_config c = cache_of(call, a[1], number32(a[7]), D, number(a[8]), pool);
    const auto qr = call.rows(q, H, D, "q");
    const double scale = a[9] == Py_None ? 1.0 / std::sqrt((double)D) : real(a[9]);
    const cs_cache_batch b = {sizeof(cs_cache_batch), (int32_t)B, T, number32(a[5]), (int32_t)width, number(a[6]),
                              static_cast<int32_t*>(call.flat(a[4], at::kInt, B + 1, "cu_queries")),
                              static_cast<int32_t*>(call.flat(a[3], at::kInt, B, "n_keys")), static_cast<int32_t*>(call.flat(table, at::kInt, B * width, "page_table"))};
    void* flag = call.optional(a[13], at::kInt, 1, "err_flag");
    size_t need = 0;
    if (const int st = cs_attention_cache_query(&c, &b, (int32_t)H, &need)) return PyLong_FromLong(st);
    at::Tensor workspace;
    if (need) {
      if (a[12] != Py_None) workspace = tensor(a[12], "workspace");
      if (!workspace.defined() || workspace.nbytes() < need) workspace = at::empty({(int64_t)need}, q.options().dtype(at::kByte));
      else if (workspace.device() != call.device || !workspace.is_contiguous()) throw Value("workspace: expected a contiguous tensor on the GPU");
    }
    const at::Tensor out = a[11] == Py_None ? at::empty({T, H, D}, q.options()) : tensor(a[11], "out");
    const auto o = call.given(out, T, H, D, at::kBFloat16, "out");
    const int st = cs_attention_cache(&c, pool, &b, qr.p, qr.row, o.p, o.row, (int32_t)H, (float)scale, truth(a[10]),
                                      need ? workspace.data_ptr() : nullptr, need, static_cast<int32_t*>(flag), call.stream());
    if (st != CS_OK) return PyLong_FromLong(st);
    return THPVariable_Wrap(out);
  });
}

// rows [rows, width] of a given type; rows may lie apart
Call::Rows matrix(const Call& call, const at::Tensor& x, int64_t n, int64_t width, at::ScalarType type, const char* name) {
  if (x.dim() != 2 || x.size(0) != n || x.size(1) != width || x.scalar_type() != type || x.device() != call.device || (n > 0 && width > 1 && x.stride(1) != 1))
    throw Value(std::string(name) + ": expected [" + std::to_string(n) + ", " + std::to_string(width) +
                "] of its type with consecutive values, on the GPU");
  return {x.data_ptr(), n > 1 ? x.stride(0) : width};        // (one row lies no distance from another)
}
void two(const at::Tensor& x, const char* name) {
  if (x.dim() != 2) throw Value(std::string(name) + ": expected [rows, width]");
}
// a size that a configuration holds in 32 bits
int32_t size32(int64_t v, const char* name) {
  if (v > 0x7fffffff) throw Value(std::string(name) + ": sizes");
  return (int32_t)v;
}
at::Tensor workspace_of(const Call& call, PyObject* given, size_t need, const at::Tensor& like) {
  at::Tensor w;
  if (!need) return w;
  if (given != Py_None) w = tensor(given, "workspace");
  if (!w.defined() || w.nbytes() < need) return at::empty({(int64_t)need}, like.options().dtype(at::kByte));
  if (w.device() != call.device || !w.is_contiguous()) throw Value("workspace: expected a contiguous tensor on the GPU");
  return w;
}

// (x, residual, pre_gain, pre_bias, post_gain, post_bias, gate, residual_scale, block_scale, norm code, eps, r, y) -> (r, y)
PyObject* norm_residual(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded(n, 13, [&]() -> PyObject* {
    const at::Tensor &x = tensor(a[0], "x"), &res = tensor(a[1], "residual");
    two(x, "x");
    const Call call(x, "x");
    const c10::DeviceGuard on(call.device);
    const int64_t T = x.size(0), W = x.size(1);
    const int code = dtype_code(x), rcode = dtype_code(res);
    cs_norm_config c = {sizeof(cs_norm_config), number32(a[9]), size32(W, "x"), code, rcode, 0, (float)real(a[10]), (float)real(a[7]), (float)real(a[8])};
    const auto xr = matrix(call, x, T, W, x.scalar_type(), "x"), rr = matrix(call, res, T, W, res.scalar_type(), "residual");
    Call::Rows gate = {nullptr, 0};
    if (a[6] != Py_None) {
      const at::Tensor& g = tensor(a[6], "gate");
      c.gate = g.dim() == 1 ? 1 : 2;
      if (c.gate == 1) gate = {call.flat(g, x.scalar_type(), W, "gate"), 0};
      else gate = matrix(call, g, T, W, x.scalar_type(), "gate");
    }
    void *pg = call.flat(a[2], at::kFloat, W, "pre_gain"), *pb = call.optional(a[3], at::kFloat, W, "pre_bias");
    void *og = call.optional(a[4], at::kFloat, W, "post_gain"), *ob = call.optional(a[5], at::kFloat, W, "post_bias");
    const at::Tensor r = a[11] == Py_None ? at::empty({T, W}, res.options()) : tensor(a[11], "r");
    const at::Tensor y = a[12] == Py_None ? at::empty({T, W}, x.options()) : tensor(a[12], "y");
    const auto rw = matrix(call, r, T, W, res.scalar_type(), "r"), yw = matrix(call, y, T, W, x.scalar_type(), "y");
    const int st = cs_norm_residual(&c, xr.p, xr.row, rr.p, rr.row, gate.p, gate.row, static_cast<float*>(og), static_cast<float*>(ob),
                                    static_cast<float*>(pg), static_cast<float*>(pb), rw.p, rw.row, yw.p, yw.row, T, call.stream());
    if (st != CS_OK) return PyLong_FromLong(st);
    PyObject *u = THPVariable_Wrap(r), *v = u ? THPVariable_Wrap(y) : nullptr, *both = v ? PyTuple_Pack(2, u, v) : nullptr;
    Py_XDECREF(u);
    Py_XDECREF(v);
    return both;
  });
}

// packed weights: (bytes tensor, format code, matrices, n, k) of the five arguments from `a` on
cs_weights_config weights_of(const Call& call, PyObject* const* a, void*& p, const char* name) {
  const cs_weights_config c = {sizeof(cs_weights_config), number32(a[1]), number(a[2]), number32(a[3]), number32(a[4])};
  size_t bytes = 0;
  if (cs_weights_query(&c, &bytes)) throw Value(std::string(name) + ": " + cs_last_error());
  p = call.flat(a[0], at::kByte, (int64_t)bytes, name);
  return c;
}

// (x, packed, format, matrices, n, k, bias, out dtype code, out, workspace) -> out
PyObject* linear_packed(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded(n, 10, [&]() -> PyObject* {
    const at::Tensor& x = tensor(a[0], "x");
    two(x, "x");
    if (x.scalar_type() != at::kBFloat16) throw Type("x must be bf16");
    const Call call(x, "x");
    const c10::DeviceGuard on(call.device);
    const int64_t T = x.size(0);
    void* packed;
    const cs_weights_config c = weights_of(call, a + 1, packed, "weights");
    const auto xr = matrix(call, x, T, c.k, at::kBFloat16, "x");
    void* bias = call.optional(a[6], at::kFloat, c.n, "bias");
    const int code = number32(a[7]);
    const at::ScalarType type = code == CS_BF16 ? at::kBFloat16 : at::kFloat;
    size_t need = 0;
    if (const int st = cs_linear_packed_query(&c, T, &need)) return PyLong_FromLong(st);
    const at::Tensor out = a[8] == Py_None ? at::empty({T, c.n}, x.options().dtype(type)) : tensor(a[8], "out");
    const auto o = matrix(call, out, T, c.n, type, "out");
    const at::Tensor workspace = workspace_of(call, a[9], need, x);
    const int st = cs_linear_packed(&c, packed, xr.p, xr.row, static_cast<float*>(bias), o.p, o.row, code, T, need ? workspace.data_ptr() : nullptr, need,
                                    call.stream());
    if (st != CS_OK) return PyLong_FromLong(st);
    return THPVariable_Wrap(out);
  });
}

// (x, router, up x 5, down x 5, top, score code, renormalise, scale, choice_bias, live, y, experts, weights, workspace) -> (y, experts, weights)
PyObject* moe(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded(n, 22, [&]() -> PyObject* {
    const at::Tensor &x = tensor(a[0], "x"), &router = tensor(a[1], "router");
    two(x, "x");
    two(router, "router");
    if (x.scalar_type() != at::kBFloat16) throw Type("x must be bf16");
    const Call call(x, "x");
    const c10::DeviceGuard on(call.device);
    const int64_t T = x.size(0), H = x.size(1), E = router.size(0);
    void *up, *down;
    const cs_weights_config u = weights_of(call, a + 2, up, "up"), d = weights_of(call, a + 7, down, "down");
    if (u.format != d.format || u.matrices != d.matrices || u.matrices < E || u.k != H || d.n != H || u.n != 2 * (int64_t)d.k)
      throw Value("up, down: expected [experts, 2 inter, hidden] and [experts, hidden, inter] of one format, the router's and shared ones");
    const int64_t top = number32(a[12]);
    if (top <= 0 || top > E) throw Value("top: expected 1 .. experts");
    const cs_moe_config c = {sizeof(cs_moe_config), u.format, size32(H, "x"), d.k, size32(E, "router"), (int32_t)(u.matrices - E), (int32_t)top, number32(a[13]),
                             truth(a[14]), (float)real(a[15])};
    const auto xr = matrix(call, x, T, H, at::kBFloat16, "x");
    void *rp = call.flat(router, at::kBFloat16, E * H, "router"), *bias = call.optional(a[16], at::kFloat, E, "choice_bias"), *live = nullptr;
    if (a[17] != Py_None) {
      const at::Tensor& l = tensor(a[17], "live");
      live = call.flat(l, l.scalar_type() == at::kByte ? at::kByte : at::kBool, T, "live");
    }
    size_t need = 0;
    if (const int st = cs_moe_query(&c, T, &need)) return PyLong_FromLong(st);
    const at::Tensor y = a[18] == Py_None ? at::empty({T, H}, x.options()) : tensor(a[18], "y");
    const at::Tensor experts = a[19] == Py_None ? at::empty({T, top}, x.options().dtype(at::kInt)) : tensor(a[19], "experts");
    const at::Tensor weights = a[20] == Py_None ? at::empty({T, top}, x.options().dtype(at::kFloat)) : tensor(a[20], "weights");
    const auto yw = matrix(call, y, T, H, at::kBFloat16, "y");
    void *ep = call.flat(experts, at::kInt, T * top, "experts"), *wp = call.flat(weights, at::kFloat, T * top, "weights");
    const at::Tensor workspace = workspace_of(call, a[21], need, x);
    const int st = cs_moe(&c, xr.p, xr.row, rp, static_cast<float*>(bias), static_cast<uint8_t*>(live), up, down, yw.p, yw.row, static_cast<int32_t*>(ep),
                          static_cast<float*>(wp), T, need ? workspace.data_ptr() : nullptr, need, call.stream());
    if (st != CS_OK) return PyLong_FromLong(st);
    PyObject *p = THPVariable_Wrap(y), *q = p ? THPVariable_Wrap(experts) : nullptr, *r = q ? THPVariable_Wrap(weights) : nullptr;
    PyObject* all = r ? PyTuple_Pack(3, p, q, r) : nullptr;
    Py_XDECREF(p);
    Py_XDECREF(q);
    Py_XDECREF(r);
    return all;
  });
}

// (packed, format, matrices, n, k, w, read, err_flag) -> None: w [matrices, n, k] is packed, or filled with what is held
PyObject* weights(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded(n, 8, [&]() -> PyObject* {
    const at::Tensor& w = tensor(a[5], "w");
    const Call call(w, "w");
    const c10::DeviceGuard on(call.device);
    void* packed;
    const cs_weights_config c = weights_of(call, a, packed, "weights");
    const int code = dtype_code(w);
    if (w.dim() != 3 || w.size(0) != c.matrices || w.size(1) != c.n || w.size(2) != c.k || (c.k > 1 && w.stride(2) != 1) || w.stride(0) < 0)
      throw Value("w: expected [matrices, n, k] with consecutive values");
    const int64_t row = c.n > 1 ? w.stride(1) : c.k;           // (one row lies no distance from another)
    void* flag = call.optional(a[7], at::kInt, 1, "err_flag");
    const int st = truth(a[6]) ? cs_weights_read(&c, packed, w.data_ptr(), row, w.stride(0), code, call.stream())
                               : cs_weights_pack(&c, w.data_ptr(), row, w.stride(0), code, packed, static_cast<int32_t*>(flag), call.stream());
    Py_INCREF(Py_None);
    return status_or(st, Py_None);
  });
}

#define CALL(name) {#name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(name)), METH_FASTCALL, nullptr}
PyMethodDef methods[] = {CALL(qk_norm_rope), CALL(cache_write), CALL(cache_read), CALL(attention_cache), CALL(norm_residual), CALL(linear_packed), CALL(moe), CALL(weights),
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_calls", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__calls() { return PyModule_Create(&module); }

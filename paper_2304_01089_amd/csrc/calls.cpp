// CPython module `_calls`: the argument marshalling of the entry points that a serving loop calls, in native code.
//
// A short call is paced by the host: a launch is 3.4 us of it, and marshalling in Python, with ctypes, was as much again (one linear
// layer, rptq_ln_quant + rptq_cluster_gemm: 15.0 us a pass).  Every function takes the binding's arguments by position and covers the
// ordinary case only: contiguous device tensors of the right type, one-dimensional float32 / int32 tables that support the buffer
// protocol, ints in range, the current stream.  For anything else it returns None without having called the library, and
// binding.py's own code converts, or raises, as it always has.  It keeps nothing between calls but the library's entry
// points and torch's stream query.
// Tensors are read through torch's C++ interface.  Asked for by their Python attributes, five of each, eleven tensors took 2.6 us more
// (rptq_rope_quant_paged of one token 7.06 -> 4.48 us a pass, rptq_attend_weights_paged of one
// sequence 7.13 -> 5.39, which the GPU takes, rptq_rope 5.16 -> 3.83, the linear layer for one row of 768 10.9 -> 9.9).
#define PY_SSIZE_T_CLEAN
#include <Python.h>
#include <stdint.h>
#include <torch/csrc/autograd/python_variable.h>

#include "rptq.h"

namespace {

decltype(&rptq_ln_quant) f_ln_quant;
decltype(&rptq_cluster_gemm) f_cluster_gemm;
decltype(&rptq_cluster_gemm_quant) f_cluster_gemm_quant;
decltype(&rptq_cluster_rowsums) f_cluster_rowsums;
decltype(&rptq_cluster_gemm_cw) f_cluster_gemm_cw;
decltype(&rptq_kv_quant) f_kv_quant;
decltype(&rptq_kv_dequant) f_kv_dequant;
decltype(&rptq_kv_page_bytes) f_kv_page_bytes;
decltype(&rptq_kv_quant_paged) f_kv_quant_paged;
decltype(&rptq_kv_dequant_paged) f_kv_dequant_paged;
decltype(&rptq_attend_paged) f_attend_paged;
decltype(&rptq_rope) f_rope;
decltype(&rptq_rope_quant_paged) f_rope_quant_paged;
decltype(&rptq_attend_weights_paged) f_attend_weights_paged;
decltype(&rptq_evict_paged) f_evict_paged;

PyObject *get_device, *get_stream;                       // torch's functions

using at::ScalarType;
constexpr ScalarType kAny = ScalarType::Undefined;       // (no tensor's type)

// Each getter returns false, with no Python error set, where the ordinary case does not apply.
bool no_error() {
  PyErr_Clear();
  return false;
}

bool get_i64(PyObject* o, int64_t* out) {
  if (!PyLong_Check(o)) return false;
  int overflow = 0;
  *out = PyLong_AsLongLongAndOverflow(o, &overflow);
  return overflow == 0;
}

bool get_i32(PyObject* o, int32_t* out) {
  int64_t v;
  if (!get_i64(o, &v) || v < INT32_MIN || v > INT32_MAX) return false;
  *out = static_cast<int32_t>(v);
  return true;
}

bool get_f32(PyObject* o, float* out) {
  if (!PyFloat_Check(o)) return false;
  *out = static_cast<float>(PyFloat_AS_DOUBLE(o));
  return true;
}

bool get_flag(PyObject* o, int32_t* out) {
  if (o != Py_True && o != Py_False) return false;
  *out = o == Py_True;
  return true;
}

// f of a tensor that is one of torch's own two classes; what has no address or no sizes throws, and is out of the ordinary.
template <typename F>
bool of_tensor(PyObject* o, F&& f) {
  if (!THPVariable_CheckExact(o)) return false;
  try {
    return f(THPVariable_Unpack(o));
  } catch (...) {
    return false;
  }
}

bool is_type(const at::Tensor& t, ScalarType type) { return type == kAny || t.scalar_type() == type; }

// Address of a contiguous device tensor of that dtype; None is NULL where it is allowed.
template <typename T>
bool get_tensor(PyObject* o, ScalarType type, bool allow_none, T** out) {
  if (o == Py_None) {
    *out = nullptr;
    return allow_none;
  }
  return of_tensor(o, [&](const at::Tensor& t) {
    if (!t.is_cuda() || !t.is_contiguous() || !is_type(t, type)) return false;
    *out = static_cast<T*>(t.data_ptr());
    return true;
  });
}

bool get_bytes(PyObject* o, int64_t* out) {
  return of_tensor(o, [&](const at::Tensor& t) {
    *out = static_cast<int64_t>(t.nbytes());
    return true;
  });
}

// A one-dimensional table of 4-byte elements ('f' or 'i'), borrowed for the call.
struct Table {
  Py_buffer b;
  bool held = false;
  ~Table() {
    if (held) PyBuffer_Release(&b);
  }
  bool get(PyObject* o, char format) {
    if (!PyObject_CheckBuffer(o)) return false;
    if (PyObject_GetBuffer(o, &b, PyBUF_C_CONTIGUOUS | PyBUF_FORMAT) != 0) return no_error();
    held = true;
    return b.ndim == 1 && b.itemsize == 4 && b.format != nullptr && b.format[0] == format && b.format[1] == 0 &&
           (reinterpret_cast<uintptr_t>(b.buf) & 3u) == 0;
  }
  const int32_t* ints() const { return static_cast<const int32_t*>(b.buf); }
  const float* floats() const { return static_cast<const float*>(b.buf); }
  int32_t size() const { return static_cast<int32_t>(b.shape[0]); }
};

bool get_current_stream(PyObject* stream, void** out) {
  if (stream != Py_None) return false;
  PyObject* device = PyObject_CallNoArgs(get_device);
  if (device == nullptr) return no_error();
  PyObject* s = PyObject_CallOneArg(get_stream, device);
  Py_DECREF(device);
  if (s == nullptr) return no_error();
  const bool ok = PyLong_Check(s);
  *out = ok ? PyLong_AsVoidPtr(s) : nullptr;
  Py_DECREF(s);
  return (ok && !PyErr_Occurred()) || no_error();
}

// Y's dtype as the library names it.
bool get_y_dtype(PyObject* y, int32_t* out) {
  return of_tensor(y, [&](const at::Tensor& t) {
    *out = t.scalar_type() == at::kFloat ? RPTQ_DTYPE_F32 : RPTQ_DTYPE_BF16;
    return t.scalar_type() == at::kFloat || t.scalar_type() == at::kBFloat16;
  });
}

template <typename F>
PyObject* run(F&& call) {                                // (other Python threads go on meanwhile, as under ctypes)
  int32_t status;
  Py_BEGIN_ALLOW_THREADS
  status = call();
  Py_END_ALLOW_THREADS
  return PyLong_FromLong(status);
}

// (x, M, d, gamma_pad, beta_pad, eps, relu, perm_pad, cluster_off, s, inv_s, z, bits, codes, xsum, rowterm, stream)
PyObject* ln_quant(PyObject*, PyObject* const* a, Py_ssize_t n) {
  void *x, *codes, *stream;
  float *gamma, *beta, *rowterm, eps;
  int32_t *perm, *xsum, d, relu, bits;
  int64_t M;
  Table off, s, inv, z;
  if (n != 17 || f_ln_quant == nullptr || !get_tensor(a[0], at::kBFloat16, false, &x) || !get_i64(a[1], &M) || !get_i32(a[2], &d) ||
      !get_tensor(a[3], at::kFloat, true, &gamma) || !get_tensor(a[4], at::kFloat, true, &beta) || !get_f32(a[5], &eps) ||
      !get_flag(a[6], &relu) || !get_tensor(a[7], at::kInt, false, &perm) || !off.get(a[8], 'i') || !s.get(a[9], 'f') ||
      !inv.get(a[10], 'f') || !z.get(a[11], 'i') || !get_i32(a[12], &bits) || !get_tensor(a[13], kAny, false, &codes) ||
      !get_tensor(a[14], at::kInt, true, &xsum) || !get_tensor(a[15], at::kFloat, true, &rowterm) || !get_current_stream(a[16], &stream))
    Py_RETURN_NONE;
  return run([&] {
    return f_ln_quant(x, M, d, gamma, beta, eps, relu, perm, off.ints(), off.size() - 1, s.floats(), inv.floats(), z.ints(),
                      bits, codes, xsum, rowterm, stream);
  });
}

// (codes, M, bits, Wq, N, cluster_off, sX, sW, zW, colterm, rowterm, y, stream)
PyObject* cluster_gemm(PyObject*, PyObject* const* a, Py_ssize_t n) {
  void *codes, *wq, *y, *stream;
  float *sw, *colterm, *rowterm;
  int32_t *zw, bits, N, y_dtype;
  int64_t M;
  Table off, sx;
  if (n != 13 || f_cluster_gemm == nullptr || !get_tensor(a[0], kAny, false, &codes) || !get_i64(a[1], &M) ||
      !get_i32(a[2], &bits) || !get_tensor(a[3], kAny, false, &wq) || !get_i32(a[4], &N) || !off.get(a[5], 'i') ||
      !sx.get(a[6], 'f') || !get_tensor(a[7], at::kFloat, false, &sw) || !get_tensor(a[8], at::kInt, false, &zw) ||
      !get_tensor(a[9], at::kFloat, false, &colterm) || !get_tensor(a[10], at::kFloat, false, &rowterm) ||
      !get_y_dtype(a[11], &y_dtype) || !get_tensor(a[11], kAny, false, &y) || !get_current_stream(a[12], &stream))
    Py_RETURN_NONE;
  return run([&] {
    return f_cluster_gemm(codes, M, bits, wq, N, off.ints(), off.size() - 1, sx.floats(), sw, zw, colterm, rowterm, y,
                          y_dtype, stream);
  });
}

// (codes, M, bits, Wq, N, cluster_off, sX, sW, zW, colterm, rowterm, relu, next_cluster_off, next_s, next_inv_s, next_z,
//  next_bits, next_codes, next_rowterm, workspace, stream)
PyObject* cluster_gemm_quant(PyObject*, PyObject* const* a, Py_ssize_t n) {
  void *codes, *wq, *next_codes, *workspace, *stream;
  float *sw, *colterm, *rowterm, *next_rowterm;
  int32_t *zw, bits, N, relu, next_bits;
  int64_t M, bytes;
  Table off, sx, noff, ns, ni, nz;
  if (n != 21 || f_cluster_gemm_quant == nullptr || !get_tensor(a[0], kAny, false, &codes) || !get_i64(a[1], &M) ||
      !get_i32(a[2], &bits) || !get_tensor(a[3], kAny, false, &wq) || !get_i32(a[4], &N) || !off.get(a[5], 'i') ||
      !sx.get(a[6], 'f') || !get_tensor(a[7], at::kFloat, false, &sw) || !get_tensor(a[8], at::kInt, false, &zw) ||
      !get_tensor(a[9], at::kFloat, false, &colterm) || !get_tensor(a[10], at::kFloat, false, &rowterm) || !get_flag(a[11], &relu) ||
      !noff.get(a[12], 'i') || !ns.get(a[13], 'f') || !ni.get(a[14], 'f') || !nz.get(a[15], 'i') ||
      !get_i32(a[16], &next_bits) || !get_tensor(a[17], kAny, false, &next_codes) ||
      !get_tensor(a[18], at::kFloat, false, &next_rowterm) || !get_tensor(a[19], kAny, false, &workspace) ||
      !get_bytes(a[19], &bytes) || !get_current_stream(a[20], &stream))
    Py_RETURN_NONE;
  return run([&] {
    return f_cluster_gemm_quant(codes, M, bits, wq, N, off.ints(), off.size() - 1, sx.floats(), sw, zw, colterm, rowterm, relu,
                                noff.ints(), noff.size() - 1, ns.floats(), ni.floats(), nz.ints(), next_bits, next_codes,
                                next_rowterm, workspace, static_cast<size_t>(bytes), stream);
  });
}

// (codes, M, bits, cluster_off, sX, zX, rowsums, stream)
PyObject* cluster_rowsums(PyObject*, PyObject* const* a, Py_ssize_t n) {
  void *codes, *stream;
  float* rowsums;
  int32_t bits;
  int64_t M;
  Table off, sx, zx;
  if (n != 8 || f_cluster_rowsums == nullptr || !get_tensor(a[0], kAny, false, &codes) || !get_i64(a[1], &M) ||
      !get_i32(a[2], &bits) || !off.get(a[3], 'i') || !sx.get(a[4], 'f') || !zx.get(a[5], 'i') ||
      !get_tensor(a[6], at::kFloat, false, &rowsums) || !get_current_stream(a[7], &stream))
    Py_RETURN_NONE;
  return run([&] { return f_cluster_rowsums(codes, M, bits, off.ints(), off.size() - 1, sx.floats(), zx.ints(), rowsums, stream); });
}

// (codes, M, bits, Wq, N, cluster_off, scale_tab, cross_tab, colterm, rowsums, y, stream)
PyObject* cluster_gemm_cw(PyObject*, PyObject* const* a, Py_ssize_t n) {
  void *codes, *wq, *y, *stream;
  float *scale, *cross, *colterm, *rowsums;
  int32_t bits, N, y_dtype;
  int64_t M;
  Table off;
  if (n != 12 || f_cluster_gemm_cw == nullptr || !get_tensor(a[0], kAny, false, &codes) || !get_i64(a[1], &M) ||
      !get_i32(a[2], &bits) || !get_tensor(a[3], kAny, false, &wq) || !get_i32(a[4], &N) || !off.get(a[5], 'i') ||
      !get_tensor(a[6], at::kFloat, false, &scale) || !get_tensor(a[7], at::kFloat, false, &cross) ||
      !get_tensor(a[8], at::kFloat, false, &colterm) || !get_tensor(a[9], at::kFloat, false, &rowsums) ||
      !get_y_dtype(a[10], &y_dtype) || !get_tensor(a[10], kAny, false, &y) || !get_current_stream(a[11], &stream))
    Py_RETURN_NONE;
  return run([&] {
    return f_cluster_gemm_cw(codes, M, bits, wq, N, off.ints(), off.size() - 1, scale, cross, colterm, rowsums, y, y_dtype, stream);
  });
}

// (x, T, d, table, bits, codes, stream) and (codes, T, d, table, bits, out, stream)
PyObject* kv_call(PyObject* const* a, Py_ssize_t n, bool quant) {
  void *from, *table, *to, *stream;
  int32_t d, bits;
  int64_t T;
  if (n != 7 || (quant ? f_kv_quant == nullptr : f_kv_dequant == nullptr) ||
      !get_tensor(a[0], quant ? at::kBFloat16 : kAny, false, &from) || !get_i64(a[1], &T) || !get_i32(a[2], &d) ||
      !get_tensor(a[3], kAny, false, &table) || !get_i32(a[4], &bits) ||
      !get_tensor(a[5], quant ? kAny : at::kBFloat16, false, &to) || !get_current_stream(a[6], &stream))
    Py_RETURN_NONE;
  return run([&] { return quant ? f_kv_quant(from, T, d, table, bits, to, stream) : f_kv_dequant(from, T, d, table, bits, to, stream); });
}
PyObject* kv_quant(PyObject*, PyObject* const* a, Py_ssize_t n) { return kv_call(a, n, true); }
PyObject* kv_dequant(PyObject*, PyObject* const* a, Py_ssize_t n) { return kv_call(a, n, false); }

// ---- the cache in pages: tensors whose sizes, strides and device count ----------------------------------
// The current device and its current stream.
bool get_place(PyObject* stream, int64_t* device, void** out) {
  if (stream != Py_None) return false;
  PyObject* d = PyObject_CallNoArgs(get_device);
  if (d == nullptr) return no_error();
  PyObject* s = PyObject_CallOneArg(get_stream, d);
  const bool ok = s != nullptr && PyLong_Check(s) && get_i64(d, device);
  *out = ok ? PyLong_AsVoidPtr(s) : nullptr;
  Py_DECREF(d);
  Py_XDECREF(s);
  return (ok && !PyErr_Occurred()) || no_error();
}

// Whether a tensor is of that dtype on that device, and its address.
template <typename T>
bool is_on(const at::Tensor& t, ScalarType type, int64_t device, T** out) {
  if (!t.is_cuda() || t.get_device() != device || !is_type(t, type)) return false;
  *out = static_cast<T*>(t.data_ptr());
  return true;
}

// A contiguous one, and how many bytes it has.
template <typename T>
bool get_whole(PyObject* o, ScalarType type, int64_t device, T** out, int64_t* bytes) {
  return of_tensor(o, [&](const at::Tensor& t) {
    *bytes = static_cast<int64_t>(t.nbytes());
    return is_on(t, type, device, out) && t.is_contiguous();
  });
}

// The sizes of a tensor of exactly so many.
bool get_sizes(PyObject* o, int n, int64_t* out) {
  return of_tensor(o, [&](const at::Tensor& t) {
    if (t.dim() != n) return false;
    for (int i = 0; i < n; ++i) out[i] = t.size(i);
    return true;
  });
}

// A two-dimensional tensor with contiguous rows, at least one of them.
struct Rows {
  void* at;
  int64_t rows, cols, ld;
  bool get(PyObject* o, ScalarType type, int64_t device) {
    return of_tensor(o, [&](const at::Tensor& t) {
      if (t.dim() != 2 || !is_on(t, type, device, &at)) return false;
      rows = t.size(0), cols = t.size(1);
      ld = rows > 1 ? t.stride(0) : cols;
      return rows >= 1 && cols >= 1 && cols <= INT32_MAX && (cols == 1 || t.stride(1) == 1);
    });
  }
};

// Both tensors' pages and tables: the same whole number of pages, and a record for each of d positions and no more (a table of
// another width is another cache's).
struct Pages {
  uint8_t *k, *v;
  void *k_table, *v_table;
  int64_t n;
  bool get(PyObject* kp, PyObject* vp, PyObject* kt, PyObject* vt, int64_t device, int64_t d, int32_t page_size, int32_t bits) {
    int64_t kb, vb, ktb, vtb;
    if (d < 1 || d > RPTQ_MAX_CHANNELS) return false;
    const int64_t size = static_cast<int64_t>(f_kv_page_bytes(static_cast<int32_t>(d), page_size, bits));
    if (size == 0 || !get_whole(kp, at::kByte, device, &k, &kb) || !get_whole(vp, at::kByte, device, &v, &vb) || kb != vb || kb < size || kb % size != 0)
      return false;
    n = kb / size;
    return get_whole(kt, kAny, device, &k_table, &ktb) && get_whole(vt, kAny, device, &v_table, &vtb) && ktb == 16 * d && vtb == 16 * d;
  }
};

bool get_slots(PyObject* t, int64_t device, int64_t rows, int64_t** out) {
  int64_t bytes, size;
  return get_whole(t, at::kLong, device, out, &bytes) && get_sizes(t, 1, &size) && size == rows;
}

// (k, v, slots, k_table, v_table, bits, k_pages, v_pages, page_size, stream)
PyObject* kv_quant_paged(PyObject*, PyObject* const* a, Py_ssize_t n) {
  Rows k, v;
  Pages p;
  int64_t device, *slots;
  int32_t bits, page_size;
  void* stream;
  if (n != 10 || f_kv_quant_paged == nullptr || !get_place(a[9], &device, &stream) || !get_i32(a[5], &bits) || !get_i32(a[8], &page_size) ||
      !k.get(a[0], at::kBFloat16, device) || !v.get(a[1], at::kBFloat16, device) || k.rows != v.rows || k.cols != v.cols ||
      !get_slots(a[2], device, k.rows, &slots) || !p.get(a[6], a[7], a[3], a[4], device, k.cols, page_size, bits))
    Py_RETURN_NONE;
  return run([&] {
    return f_kv_quant_paged(k.at, k.ld, v.at, v.ld, k.rows, static_cast<int32_t>(k.cols), p.k_table, p.v_table, bits, slots, p.k, p.v, p.n,
                            page_size, stream);
  });
}

// (k_pages, v_pages, page_size, bits, slots, k_table, v_table, k, v, stream)
PyObject* kv_dequant_paged(PyObject*, PyObject* const* a, Py_ssize_t n) {
  Rows k, v;
  Pages p;
  int64_t device, *slots;
  int32_t bits, page_size;
  void* stream;
  if (n != 10 || f_kv_dequant_paged == nullptr || !get_place(a[9], &device, &stream) || !get_i32(a[3], &bits) || !get_i32(a[2], &page_size) ||
      !k.get(a[7], at::kBFloat16, device) || !v.get(a[8], at::kBFloat16, device) || k.rows != v.rows || k.cols != v.cols ||
      !get_slots(a[4], device, k.rows, &slots) || !p.get(a[0], a[1], a[5], a[6], device, k.cols, page_size, bits))
    Py_RETURN_NONE;
  return run([&] {
    return f_kv_dequant_paged(p.k, p.v, p.n, page_size, bits, slots, k.rows, static_cast<int32_t>(k.cols), p.k_table, p.v_table, k.at, k.ld,
                              v.at, v.ld, stream);
  });
}

// (q, n_q_heads, n_kv_heads, head_dim, scale, k_table, v_table, bits, k_pages, v_pages, page_size, page_table, lens, out, lse, workspace, stream)
PyObject* attend_paged(PyObject*, PyObject* const* a, Py_ssize_t n) {
  Rows q, table, out;
  Pages p;
  int64_t device, lens_bytes, lse_bytes = 0, ws_bytes, b;
  int32_t n_q, n_kv, hd, bits, page_size, *lens, out_dtype;
  float scale, *lse = nullptr;
  void *workspace, *stream;
  if (n != 17 || f_attend_paged == nullptr || !get_place(a[16], &device, &stream) || !get_i32(a[1], &n_q) || !get_i32(a[2], &n_kv) ||
      !get_i32(a[3], &hd) || !get_f32(a[4], &scale) || !get_i32(a[7], &bits) || !get_i32(a[10], &page_size) || n_q < 1 || n_kv < 1 || hd < 1 ||
      !q.get(a[0], at::kBFloat16, device) || q.cols != static_cast<int64_t>(n_q) * hd || q.rows > INT32_MAX)
    Py_RETURN_NONE;
  if (!p.get(a[8], a[9], a[5], a[6], device, static_cast<int64_t>(n_kv) * hd, page_size, bits) || !get_y_dtype(a[13], &out_dtype) ||
      !out.get(a[13], kAny, device) || out.rows != q.rows || out.cols != q.cols || !table.get(a[11], at::kInt, device) ||
      table.rows != q.rows || !get_whole(a[12], at::kInt, device, &lens, &lens_bytes) ||
      !get_sizes(a[12], 1, &b) || b != q.rows || !get_whole(a[15], kAny, device, &workspace, &ws_bytes))
    Py_RETURN_NONE;
  if (a[14] != Py_None && (!get_whole(a[14], at::kFloat, device, &lse, &lse_bytes) || lse_bytes < 4 * q.rows * n_q)) Py_RETURN_NONE;
  return run([&] {
    return f_attend_paged(q.at, q.ld, static_cast<int32_t>(q.rows), n_q, n_kv, hd, scale, p.k_table, p.v_table, bits, p.k, p.v, p.n,
                          page_size, static_cast<int32_t*>(table.at), table.ld, static_cast<int32_t>(table.cols), lens, out.at, out.ld,
                          out_dtype, lse, workspace, static_cast<size_t>(ws_bytes), stream);
  });
}

bool get_f64(PyObject* o, double* out) {
  if (!PyFloat_Check(o)) return false;
  *out = PyFloat_AS_DOUBLE(o);
  return true;
}

// A contiguous tensor with one entry of that type per row.
template <typename T>
bool get_column(PyObject* t, ScalarType dtype, int64_t device, int64_t rows, T** out) {
  int64_t bytes, size;
  return get_whole(t, dtype, device, out, &bytes) && get_sizes(t, 1, &size) && size == rows;
}

// The arguments of a rotation: (head_dim, rotary_dim, interleaved, freqs, amplitude).
struct Turn {
  int32_t hd, rot, interleaved;
  double *freqs, amplitude;
  bool get(PyObject* const* a, int64_t device) {
    return get_i32(a[0], &hd) && get_i32(a[1], &rot) && get_flag(a[2], &interleaved) && hd >= 1 && rot >= 2 && rot % 2 == 0 &&
           get_column(a[3], at::kDouble, device, rot / 2, &freqs) && get_f64(a[4], &amplitude);
  }
};

// (x, y, positions, head_dim, rotary_dim, interleaved, freqs, amplitude, stream)
PyObject* rope(PyObject*, PyObject* const* a, Py_ssize_t n) {
  Rows x, y;
  Turn t;
  int64_t device;
  int32_t *positions, x_dtype, y_dtype;
  void* stream;
  if (n != 9 || f_rope == nullptr || !get_place(a[8], &device, &stream) || !get_y_dtype(a[0], &x_dtype) || !get_y_dtype(a[1], &y_dtype) ||
      !x.get(a[0], kAny, device) || !y.get(a[1], kAny, device) || x.rows != y.rows || x.cols != y.cols ||
      !get_column(a[2], at::kInt, device, x.rows, &positions) || !t.get(a + 3, device) || x.cols % t.hd != 0)
    Py_RETURN_NONE;
  return run([&] {
    return f_rope(x.at, x_dtype, x.ld, y.at, y_dtype, y.ld, positions, x.rows, static_cast<int32_t>(x.cols / t.hd), t.hd, t.rot, t.interleaved,
                  t.freqs, t.amplitude, stream);
  });
}

// (q, q_out, k, v, positions, slots, head_dim, rotary_dim, interleaved, freqs, amplitude, k_table, v_table, bits, k_pages, v_pages, page_size,
//  stream)
PyObject* rope_quant_paged(PyObject*, PyObject* const* a, Py_ssize_t n) {
  Rows q{}, out{}, k, v;
  Pages p;
  Turn t;
  int64_t device, *slots;
  int32_t *positions, bits, page_size;
  void* stream;
  if (n != 18 || f_rope_quant_paged == nullptr || !get_place(a[17], &device, &stream) || !get_i32(a[13], &bits) || !get_i32(a[16], &page_size) ||
      !k.get(a[2], at::kBFloat16, device) || !v.get(a[3], at::kBFloat16, device) || k.rows != v.rows || k.cols != v.cols ||
      !get_column(a[4], at::kInt, device, k.rows, &positions) || !get_slots(a[5], device, k.rows, &slots) || !t.get(a + 6, device) ||
      k.cols % t.hd != 0 || !p.get(a[14], a[15], a[11], a[12], device, k.cols, page_size, bits))
    Py_RETURN_NONE;
  if (a[0] != Py_None || a[1] != Py_None) {
    if (!q.get(a[0], at::kBFloat16, device) || !out.get(a[1], at::kBFloat16, device) || q.rows != k.rows || out.rows != q.rows || out.cols != q.cols ||
        q.cols % t.hd != 0)
      Py_RETURN_NONE;
  }
  return run([&] {
    return f_rope_quant_paged(q.at, q.ld, out.at, out.ld, static_cast<int32_t>(q.cols / t.hd), k.at, k.ld, v.at, v.ld, k.rows,
                              static_cast<int32_t>(k.cols / t.hd), t.hd, positions, t.rot, t.interleaved, t.freqs, t.amplitude, p.k_table,
                              p.v_table, bits, slots, p.k, p.v, p.n, page_size, stream);
  });
}

// Both tensors [B, heads, capacity] of a record of every token.
struct Records {
  float* weights;
  int32_t* positions;
  int64_t capacity;
  bool get(PyObject* w, PyObject* pos, int64_t device, int64_t B, int64_t heads) {
    int64_t bytes, a[3], b[3];
    if (!get_whole(w, at::kFloat, device, &weights, &bytes) || !get_whole(pos, at::kInt, device, &positions, &bytes) ||
        !get_sizes(w, 3, a) || !get_sizes(pos, 3, b))
      return false;
    capacity = a[2];
    return a[0] == B && a[1] == heads && b[0] == B && b[1] == heads && b[2] == capacity && capacity >= 1;
  }
};

// (q, queries, n_q_heads, n_kv_heads, head_dim, scale, k_table, bits, k_pages, page_size, page_table, lens, lse, positions, fresh, weights,
//  token_positions, workspace, stream)
PyObject* attend_weights_paged(PyObject*, PyObject* const* a, Py_ssize_t n) {
  Rows q, table;
  Pages p;
  Records w;
  int64_t device, lse_bytes, shape[2], ws_bytes = 0;
  int32_t queries, n_q, n_kv, hd, bits, page_size, fresh, *lens, *positions = nullptr;
  float scale, *lse;
  void *stream, *workspace = nullptr;
  if (n != 19 || f_attend_weights_paged == nullptr || !get_place(a[18], &device, &stream) || !get_i32(a[1], &queries) || !get_i32(a[2], &n_q) ||
      !get_i32(a[3], &n_kv) || !get_i32(a[4], &hd) || !get_f32(a[5], &scale) || !get_i32(a[7], &bits) || !get_i32(a[9], &page_size) ||
      !get_i32(a[14], &fresh) || queries < 1 || n_q < 1 || n_kv < 1 || hd < 1 || !q.get(a[0], at::kBFloat16, device) ||
      q.cols != static_cast<int64_t>(n_q) * hd || !table.get(a[10], at::kInt, device) || table.rows > INT32_MAX || q.rows != table.rows * queries)
    Py_RETURN_NONE;
  if (!p.get(a[8], a[8], a[6], a[6], device, static_cast<int64_t>(n_kv) * hd, page_size, bits) || !get_column(a[11], at::kInt, device, table.rows, &lens) ||
      !get_whole(a[12], at::kFloat, device, &lse, &lse_bytes) || !get_sizes(a[12], 2, shape) || shape[0] != q.rows ||
      shape[1] != n_q || !w.get(a[15], a[16], device, table.rows, n_kv))
    Py_RETURN_NONE;
  if (a[13] != Py_None && !get_column(a[13], at::kInt, device, table.rows, &positions)) Py_RETURN_NONE;
  if (a[17] != Py_None && !get_whole(a[17], kAny, device, &workspace, &ws_bytes)) Py_RETURN_NONE;
  return run([&] {
    return f_attend_weights_paged(q.at, q.ld, static_cast<int32_t>(table.rows), queries, n_q, n_kv, hd, scale, p.k_table, bits, p.k, p.n, page_size,
                                  static_cast<int32_t*>(table.at), table.ld, static_cast<int32_t>(table.cols), lens, lse, positions, fresh,
                                  w.weights, w.positions, w.capacity, workspace, static_cast<size_t>(ws_bytes), stream);
  });
}

// (n_kv_heads, head_dim, bits, k_pages, v_pages, page_size, page_table, lens, weights, token_positions, budget, first, recent, weights_out,
//  token_positions_out, lens_out, workspace, stream)
PyObject* evict_paged(PyObject*, PyObject* const* a, Py_ssize_t n) {
  Rows table;
  Records w, out;
  int64_t device, kb, vb, ws_bytes;
  int32_t n_kv, hd, bits, page_size, budget, first, recent, *lens, *lens_out;
  uint8_t *k, *v;
  void *workspace, *stream;
  if (n != 18 || f_evict_paged == nullptr || !get_place(a[17], &device, &stream) || !get_i32(a[0], &n_kv) || !get_i32(a[1], &hd) ||
      !get_i32(a[2], &bits) || !get_i32(a[5], &page_size) || !get_i32(a[10], &budget) || !get_i32(a[11], &first) || !get_i32(a[12], &recent) ||
      n_kv < 1 || hd < 1 || static_cast<int64_t>(n_kv) * hd > RPTQ_MAX_CHANNELS || !table.get(a[6], at::kInt, device) || table.rows > INT32_MAX)
    Py_RETURN_NONE;
  const int64_t size = static_cast<int64_t>(f_kv_page_bytes(n_kv * hd, page_size, bits));
  if (size == 0 || !get_whole(a[3], at::kByte, device, &k, &kb) || !get_whole(a[4], at::kByte, device, &v, &vb) || kb != vb || kb < size || kb % size != 0 ||
      !get_column(a[7], at::kInt, device, table.rows, &lens) || !get_column(a[15], at::kInt, device, table.rows, &lens_out) ||
      !w.get(a[8], a[9], device, table.rows, n_kv) || !out.get(a[13], a[14], device, table.rows, n_kv) || out.capacity != w.capacity ||
      !get_whole(a[16], kAny, device, &workspace, &ws_bytes))
    Py_RETURN_NONE;
  return run([&] {
    return f_evict_paged(static_cast<int32_t>(table.rows), n_kv, hd, bits, k, v, kb / size, page_size, static_cast<int32_t*>(table.at), table.ld,
                         static_cast<int32_t>(table.cols), lens, w.weights, w.positions, w.capacity, budget, first, recent, out.weights,
                         out.positions, lens_out, workspace, static_cast<size_t>(ws_bytes), stream);
  });
}

template <typename F>
bool set_entry(PyObject* addresses, const char* name, F* f) {
  PyObject* o = PyDict_GetItemString(addresses, name);   // (borrowed)
  if (o == nullptr) {
    PyErr_Format(PyExc_KeyError, "%s", name);
    return false;
  }
  void* p = PyLong_AsVoidPtr(o);
  *f = reinterpret_cast<F>(p);
  return !PyErr_Occurred();
}

// setup({entry point: address}, {name: torch object}): called whenever a library is loaded.
PyObject* setup(PyObject*, PyObject* args) {
  PyObject *addresses, *objects;
  if (!PyArg_ParseTuple(args, "O!O!", &PyDict_Type, &addresses, &PyDict_Type, &objects)) return nullptr;
  const struct { const char* name; PyObject** at; } wanted[] = {{"get_device", &get_device}, {"get_stream", &get_stream}};
  for (const auto& w : wanted) {
    PyObject* o = PyDict_GetItemString(objects, w.name);
    if (o == nullptr) return PyErr_Format(PyExc_KeyError, "%s", w.name);
    Py_INCREF(o);
    Py_XSETREF(*w.at, o);
  }
  if (!set_entry(addresses, "rptq_ln_quant", &f_ln_quant) || !set_entry(addresses, "rptq_cluster_gemm", &f_cluster_gemm) ||
      !set_entry(addresses, "rptq_cluster_gemm_quant", &f_cluster_gemm_quant) ||
      !set_entry(addresses, "rptq_cluster_rowsums", &f_cluster_rowsums) ||
      !set_entry(addresses, "rptq_cluster_gemm_cw", &f_cluster_gemm_cw) || !set_entry(addresses, "rptq_kv_quant", &f_kv_quant) ||
      !set_entry(addresses, "rptq_kv_dequant", &f_kv_dequant) || !set_entry(addresses, "rptq_kv_page_bytes", &f_kv_page_bytes) ||
      !set_entry(addresses, "rptq_kv_quant_paged", &f_kv_quant_paged) ||
      !set_entry(addresses, "rptq_kv_dequant_paged", &f_kv_dequant_paged) || !set_entry(addresses, "rptq_attend_paged", &f_attend_paged) ||
      !set_entry(addresses, "rptq_rope", &f_rope) || !set_entry(addresses, "rptq_rope_quant_paged", &f_rope_quant_paged) ||
      !set_entry(addresses, "rptq_attend_weights_paged", &f_attend_weights_paged) ||
      !set_entry(addresses, "rptq_evict_paged", &f_evict_paged))
    return nullptr;
  Py_RETURN_NONE;
}

#define RPTQ_METHOD(name) {#name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(name)), METH_FASTCALL, nullptr}
PyMethodDef methods[] = {RPTQ_METHOD(ln_quant), RPTQ_METHOD(cluster_gemm), RPTQ_METHOD(cluster_gemm_quant),
                         RPTQ_METHOD(cluster_rowsums), RPTQ_METHOD(cluster_gemm_cw), RPTQ_METHOD(kv_quant),
                         RPTQ_METHOD(kv_dequant), RPTQ_METHOD(kv_quant_paged), RPTQ_METHOD(kv_dequant_paged),
                         RPTQ_METHOD(attend_paged), RPTQ_METHOD(rope), RPTQ_METHOD(rope_quant_paged), RPTQ_METHOD(attend_weights_paged),
                         RPTQ_METHOD(evict_paged), {"setup", setup, METH_VARARGS, nullptr}, {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_calls", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__calls(void) {
  PyObject* m = PyModule_Create(&module);
  // (torch.__version__ of the torch that it was built with, before and behind the plus)
  if (m != nullptr && (PyModule_AddStringConstant(m, "torch_version", RPTQ_TORCH_VERSION) != 0 ||
                       PyModule_AddStringConstant(m, "torch_local", RPTQ_TORCH_LOCAL) != 0))
    Py_CLEAR(m);
  return m;
}

// Tensor arguments of the calls that take a few microseconds (rotary table, norms and rotation, int8 rows and
// products, quantised cache): checks types, shapes, strides and devices, fills the C structs and makes the call.  In
// Python the same attribute reads cost about 4 us a call, as much as the launch; here 0.3 us.  Nothing is
// computed or kept.  The library's functions come as addresses from the ctypes binding (init), so there is one copy
// of it in the process.
#include <Python.h>

#include <algorithm>
#include <exception>

#include <torch/csrc/autograd/python_variable.h>

#include "../include/dc.h"

namespace {

decltype(&dc_rope_table) f_rope_table;
decltype(&dc_qk_norm_rope) f_qk_norm_rope;
decltype(&dc_quantize_rows) f_quantize_rows;
decltype(&dc_linear_i8) f_linear_i8;
decltype(&dc_cache_store_q) f_cache_store_q;
decltype(&dc_cache_apply_q) f_cache_apply_q;

// A refusal: becomes a ValueError (or keeps the Python error that is set).
struct Refused {};
[[noreturn]] void refuse(const char* what) {
  PyErr_SetString(PyExc_ValueError, what);
  throw Refused{};
}
void need(bool ok, const char* what) {
  if (!ok) refuse(what);
}

// One call's tensors, all on GPU `device`.
struct Args {
  PyObject* const* a;
  int64_t device;
  hipStream_t stream;
  // The last two arguments of every call: the tensors' device and the stream's handle.
  Args(PyObject* const* args, Py_ssize_t got, Py_ssize_t wanted) : a(args) {
    need(got == wanted, "wrong number of arguments");
    device = whole_number(a[wanted - 2]);
    const unsigned long long h = PyLong_AsUnsignedLongLong(a[wanted - 1]);
    if (PyErr_Occurred()) throw Refused{};
    stream = reinterpret_cast<hipStream_t>(h);
  }
  static int64_t whole_number(PyObject* o) {
    const long long v = PyLong_AsLongLong(o);
    if (v == -1 && PyErr_Occurred()) throw Refused{};
    return v;
  }
  double number(int i) const {
    const double v = PyFloat_AsDouble(a[i]);
    if (v == -1.0 && PyErr_Occurred()) throw Refused{};
    return v;
  }
  bool truth(int i) const {
    const int v = PyObject_IsTrue(a[i]);
    if (v < 0) throw Refused{};
    return v != 0;
  }
  const at::Tensor& tensor(int i) const {
    need(THPVariable_Check(a[i]), "a tensor is wanted");
    const at::Tensor& t = THPVariable_Unpack(a[i]);
    need(t.get_device() == device, "tensors must be on one GPU");          // -1: the host
    return t;
  }
  const at::Tensor* maybe(int i) const { return a[i] == Py_None ? nullptr : &tensor(i); }
  template <class T>
  static T* at(const at::Tensor* t) { return t ? static_cast<T*>(t->data_ptr()) : nullptr; }

  // a ctypes struct of the size of T
  template <class T>
  T structure(int i, const char* what) const {
    Py_buffer b;
    if (PyObject_GetBuffer(a[i], &b, PyBUF_SIMPLE)) throw Refused{};
    const bool ok = b.len == Py_ssize_t(sizeof(T));
    T v{};
    if (ok) v = *static_cast<const T*>(b.buf);
    PyBuffer_Release(&b);
    need(ok, what);
    return v;
  }
  dc_model_cfg cfg(int i) const {
    const dc_model_cfg c = structure<dc_model_cfg>(i, "cfg: a ModelCfg is wanted");
    need(c.patch > 0, "cfg: patch must be positive");
    return c;
  }
  // float32 [n], contiguous
  const float* vector(int i, int64_t n, const char* what) const {
    const at::Tensor* t = maybe(i);
    need(!t || (t->scalar_type() == at::kFloat && t->dim() == 1 && t->size(0) == n && t->is_contiguous()), what);
    return at<float>(t);
  }
  // the samples, inside a batch of `batch`
  int samples(int i, int64_t batch, int32_t (&out)[DC_MAX_BATCH]) const {
    PyObject* const s = PySequence_Fast(a[i], "idx: a sequence of sample indices is wanted");
    if (!s) throw Refused{};
    const Py_ssize_t n = PySequence_Fast_GET_SIZE(s);
    bool ok = n <= DC_MAX_BATCH, error = false;
    for (Py_ssize_t j = 0; ok && !error && j < n; ++j) {
      if (j >= PySequence_Fast_GET_SIZE(s)) {         // an item's __index__ may change the list
        ok = false;
        break;
      }
      const Py_ssize_t v = PyNumber_AsSsize_t(PySequence_Fast_GET_ITEM(s, j), PyExc_ValueError);
      if (v == -1 && PyErr_Occurred()) error = true;
      ok = v >= 0 && v < batch;
      out[j] = int32_t(v);
    }
    Py_DECREF(s);
    if (error) throw Refused{};
    need(ok, "idx: samples inside the batch, at most DC_MAX_BATCH of them, are wanted");
    return int(n);
  }
};

int64_t video_tokens(const dc_model_cfg& c) { return int64_t(c.lat_t) * (c.lat_h / c.patch) * (c.lat_w / c.patch); }

// [n0, n1, n2] of the type, contiguous; n0 < 0: any
void whole(const at::Tensor& t, at::ScalarType type, int64_t n0, int64_t n1, int64_t n2, const char* what) {
  need(t.scalar_type() == type && t.dim() == 3 && (n0 < 0 || t.size(0) == n0) && t.size(1) == n1 && t.size(2) == n2 &&
           t.is_contiguous(), what);
}

// Row stride of a 2-d tensor whose rows are contiguous and apart.
int64_t rows(const at::Tensor& t, const char* what) {
  need(t.dim() == 2, what);
  const int64_t n = t.size(0), cols = t.size(1);
  const int64_t ld = n <= 1 ? cols : t.stride(0);              // one row: any stride
  need((cols <= 1 || t.stride(1) == 1) && ld >= cols, what);
  return ld;
}
// The same of [B, N, width] rows that are equally far apart (a dimension of one says nothing), `wanted` of their values
// read or written.
int64_t sample_rows(const at::Tensor& t, int64_t tokens, int64_t wanted, const char* what) {
  need(t.dim() == 3 && t.size(1) == tokens && t.size(2) >= wanted && t.stride(2) == 1, what);
  const int64_t batch = t.size(0);
  const int64_t ld = tokens > 1 ? t.stride(1) : batch > 1 ? t.stride(0) : wanted;
  need((tokens * batch <= 1 || ld >= wanted) && (tokens <= 1 || batch <= 1 || t.stride(0) == tokens * ld), what);
  return ld;
}
// `n` rows of `width` bytes, `ld` bytes apart (at least the width).
struct Span {
  const char* p;
  int64_t n, ld, width;
  Span(const void* at, int64_t rows, int64_t ld_bytes, int64_t width_bytes)
      : p(static_cast<const char*>(at)), n(rows), ld(ld_bytes), width(width_bytes) {}
  explicit Span(const at::Tensor& t) : Span(t.data_ptr(), 1, int64_t(t.nbytes()), int64_t(t.nbytes())) {}      // contiguous
  const char* end() const { return p + (n - 1) * ld + width; }
};
bool overlap(const Span& a, const Span& b) {
  if (a.n < 1 || b.n < 1 || a.width < 1 || b.width < 1 || a.end() <= b.p || b.end() <= a.p) return false;
  if (a.ld == b.ld) {                   // side by side in rows of one length
    const int64_t d = (b.p - a.p) % a.ld, at = d < 0 ? d + a.ld : d;
    return at < a.width || at + b.width > a.ld;
  }
  const char *x = a.p, *y = b.p;
  for (int64_t i = 0, j = 0; i < a.n && j < b.n;) {
    if (x + a.width <= y) ++i, x += a.ld;
    else if (y + b.width <= x) ++j, y += b.ld;
    else return true;
  }
  return false;
}
int32_t dtype(const at::Tensor& t) {
  if (t.scalar_type() == at::kFloat) return DC_F32;
  need(t.scalar_type() == at::kBFloat16, "float32 or bfloat16 tensors only");
  return DC_BF16;
}
int32_t i32(int64_t v) {
  need(v <= INT32_MAX, "a size exceeds 2^31");
  return int32_t(v);
}

// The C call without the interpreter's lock; its status.
struct Unlocked {                       // taken again also when a tensor's pointer throws
  PyThreadState* const state = PyEval_SaveThread();
  ~Unlocked() { PyEval_RestoreThread(state); }
};
template <class F>
PyObject* call(const Args& a, F&& f) {
  need(a.device >= 0, "tensors must be on a GPU");
  dc_status rc;
  {
    Unlocked u;
    rc = f();
  }
  return PyLong_FromLong(rc);
}

PyObject* rope_table(PyObject* const* args, Py_ssize_t n) {          // cfg, axes, pos, table
  const Args a(args, n, 6);
  const dc_model_cfg c = a.cfg(0);
  const dc_rope_axes axes = a.structure<dc_rope_axes>(1, "axes: a RopeAxes is wanted");
  const at::Tensor* pos = a.maybe(2);
  const at::Tensor& table = a.tensor(3);
  const int64_t nv = video_tokens(c);
  whole(table, at::kFloat, nv, c.head_dim / 2, 2, "table: a contiguous float32 [N_v, head_dim / 2, 2] tensor is wanted");
  need(!pos || (pos->scalar_type() == at::kDouble && pos->dim() == 2 && pos->size(0) == nv && pos->size(1) == 3 &&
                pos->is_contiguous()), "pos: a contiguous float64 [N_v, 3] tensor or None is wanted");
  return call(a, [&] { return f_rope_table(&c, &axes, a.at<double>(pos), a.at<float>(&table), a.stream); });
}

// cfg, x, out, idx, q_weight, k_weight, eps, table, interleaved, q_scale
PyObject* qk_norm_rope(PyObject* const* args, Py_ssize_t n) {
  const Args a(args, n, 12);
  const dc_model_cfg c = a.cfg(0);
  const at::Tensor &x = a.tensor(1), &out = a.tensor(2);
  const int64_t nv = video_tokens(c), tokens = nv + c.n_txt, d2 = 2 * int64_t(c.hidden);
  const at::ScalarType type = c.dtype == DC_BF16 ? at::kBFloat16 : at::kFloat;
  const char* of_rows = "x and out: [B, N, at least 2 hidden] tensors of the model's dtype with equally spaced rows are wanted";
  need(x.scalar_type() == type && out.scalar_type() == type, of_rows);
  const int64_t ld_x = sample_rows(x, tokens, d2, of_rows), ld_out = sample_rows(out, tokens, d2, of_rows);
  dc_qk_cfg q{};
  q.q_weight = a.vector(4, c.head_dim, "q_weight: a contiguous float32 [head_dim] tensor is wanted");
  q.k_weight = a.vector(5, c.head_dim, "k_weight: a contiguous float32 [head_dim] tensor is wanted");
  q.eps = float(a.number(6));
  const at::Tensor* table = a.maybe(7);
  if (table)
    whole(*table, at::kFloat, nv, c.head_dim / 2, 2, "table: a contiguous float32 [N_v, head_dim / 2, 2] tensor is wanted");
  q.cos_sin = a.at<float>(table);
  q.interleaved = a.truth(8) ? 1 : 0;
  const float scale = float(a.number(9));
  int32_t idx[DC_MAX_BATCH];
  const int k = a.samples(3, std::min(x.size(0), out.size(0)), idx);
  const int64_t e = x.element_size();
  const Span from(x.data_ptr(), x.size(0) * tokens, ld_x * e, d2 * e);
  const Span to(out.data_ptr(), out.size(0) * tokens, ld_out * e, d2 * e);
  need((from.p == to.p && from.ld == to.ld) || !overlap(from, to), "out overlaps x: x itself, or other rows or columns, are wanted");
  return call(a, [&] {
    return f_qk_norm_rope(&c, &q, x.data_ptr(), ld_x, out.data_ptr(), ld_out, scale, idx, k, a.stream);
  });
}

PyObject* quantize_rows(PyObject* const* args, Py_ssize_t n) {       // x, q, scale
  const Args a(args, n, 5);
  const at::Tensor &x = a.tensor(0), &q = a.tensor(1);
  const int64_t ldx = rows(x, "x: a 2-d tensor with contiguous rows that do not overlap is wanted");
  const int64_t ldq = rows(q, "q: a 2-d tensor with contiguous rows that do not overlap is wanted");
  const int64_t m = x.size(0), cols = x.size(1);
  need(q.scalar_type() == at::kChar && q.size(0) == m && q.size(1) >= (cols + 127) / 128 * 128,
       "q: an int8 tensor of x's rows, at least cols rounded up to 128 wide, is wanted");
  a.tensor(2);
  const float* scale = a.vector(2, m, "scale: a contiguous float32 [rows] tensor is wanted");
  const int32_t type = dtype(x), rows32 = i32(m), cols32 = i32(cols);
  const Span from(x.data_ptr(), m, ldx * x.element_size(), cols * x.element_size());
  const Span to(q.data_ptr(), m, ldq, (cols + 127) / 128 * 128), scales(a.tensor(2));
  need(!overlap(to, from) && !overlap(scales, from) && !overlap(scales, to), "x, q and scale overlap");
  return call(a, [&] {
    return f_quantize_rows(x.data_ptr(), type, ldx, rows32, cols32, static_cast<int8_t*>(q.data_ptr()), ldq,
                           const_cast<float*>(scale), a.stream);
  });
}

PyObject* linear_i8(PyObject* const* args, Py_ssize_t n) {  // x, x_scale, w, w_scale, out, bias, gelu, gate, residual
  const Args a(args, n, 11);
  const at::Tensor &x = a.tensor(0), &w = a.tensor(2), &out = a.tensor(4);
  const char* two_d = "x, w, out and residual: 2-d tensors with contiguous rows that do not overlap are wanted";
  dc_linear_i8_args p{};
  p.ld_x = rows(x, two_d);
  p.ld_w = rows(w, two_d);
  p.ld_out = rows(out, two_d);
  const int64_t m = x.size(0), k = x.size(1), cols = w.size(0);
  need(x.scalar_type() == at::kChar && w.scalar_type() == at::kChar && w.size(1) == k,
       "x and w: int8 tensors of equally long rows are wanted");
  need(out.size(0) == m && out.size(1) == cols, "out: a [rows of x, rows of w] tensor is wanted");
  a.tensor(1);
  a.tensor(3);
  p.rows = i32(m);
  p.out_features = i32(cols);
  p.in_features = i32(k);
  p.x = static_cast<const int8_t*>(x.data_ptr());
  p.w = static_cast<const int8_t*>(w.data_ptr());
  p.out = out.data_ptr();
  p.out_dtype = dtype(out);
  p.x_scale = a.vector(1, m, "x_scale: a contiguous float32 [rows of x] tensor is wanted");
  p.w_scale = a.vector(3, cols, "w_scale: a contiguous float32 [rows of w] tensor is wanted");
  p.bias = a.vector(5, cols, "bias: a contiguous float32 [rows of w] tensor is wanted");
  p.gelu = a.truth(6) ? 1 : 0;
  p.gate = a.vector(7, cols, "gate: a contiguous float32 [rows of w] tensor is wanted");
  if (const at::Tensor* r = a.maybe(8)) {
    p.ld_residual = rows(*r, two_d);
    need(r->scalar_type() == at::kFloat && r->size(0) == m && r->size(1) == cols,
         "residual: a float32 tensor of out's shape is wanted");
    p.residual = a.at<float>(r);
  }
  const int64_t e = out.element_size();
  const Span to(out.data_ptr(), m, p.ld_out * e, cols * e);
  bool apart = !overlap(to, Span(p.x, m, p.ld_x, k)) && !overlap(to, Span(p.w, cols, p.ld_w, k));
  for (const int i : {1, 3, 5, 7})
    if (const at::Tensor* t = a.maybe(i)) apart = apart && !overlap(to, Span(*t));
  if (p.residual && !(p.residual == p.out && p.ld_residual == p.ld_out))
    apart = apart && !overlap(to, Span(p.residual, m, p.ld_residual * 4, cols * 4));
  need(apart, "out overlaps another operand: the residual itself, or other rows or columns, are wanted");
  return call(a, [&] { return f_linear_i8(&p, a.stream); });
}

// cfg, bits, first, second, codes, scales, idx: first and second are h_out and h_in (store) or h_in and g (apply)
template <bool STORE>
PyObject* cache_q(PyObject* const* args, Py_ssize_t n) {
  const Args a(args, n, 9);
  const dc_model_cfg c = a.cfg(0);
  const int64_t bits = a.whole_number(a.a[1]);
  need(bits == 8 || bits == 4, "bits must be 8 or 4");
  const at::Tensor &f = a.tensor(2), &g = a.tensor(3), &codes = a.tensor(4), &scales = a.tensor(5);
  const int64_t nv = video_tokens(c), tokens = nv + c.n_txt, d = c.hidden;
  for (const at::Tensor* t : {&f, &g})
    whole(*t, at::kFloat, -1, tokens, d, "h_in, h_out and g: contiguous float32 [B, N, hidden] tensors are wanted");
  whole(codes, bits == 8 ? at::kChar : at::kByte, -1, nv, d * bits / 8,
        "codes: a contiguous int8 [B, N_v, hidden] or (4 bits) uint8 [B, N_v, hidden / 2] tensor is wanted");
  whole(scales, at::kFloat, -1, nv, d / 64, "scales: a contiguous float32 [B, N_v, hidden / 64] tensor is wanted");
  int32_t idx[DC_MAX_BATCH];
  const int k = a.samples(6, std::min(std::min(f.size(0), g.size(0)), std::min(codes.size(0), scales.size(0))), idx);
  return call(a, [&] {
    if (STORE)
      return f_cache_store_q(&c, int32_t(bits), a.at<float>(&f), a.at<float>(&g), codes.data_ptr(), a.at<float>(&scales),
                             idx, k, a.stream);
    return f_cache_apply_q(&c, int32_t(bits), a.at<float>(&f), codes.data_ptr(), a.at<float>(&scales), a.at<float>(&g),
                           idx, k, a.stream);
  });
}

template <PyObject* (*F)(PyObject* const*, Py_ssize_t)>
PyObject* entry(PyObject*, PyObject* const* args, Py_ssize_t n) {
  try {
    return F(args, n);
  } catch (const Refused&) {
    return nullptr;
  } catch (const std::exception& e) {
    PyErr_SetString(PyExc_RuntimeError, e.what());
    return nullptr;
  }
}

// addresses of the library's functions, in the order of the pointers above
PyObject* init(PyObject*, PyObject* const* args, Py_ssize_t n) {
  void* p[6];
  if (n != 6) {
    PyErr_SetString(PyExc_ValueError, "six addresses are wanted");
    return nullptr;
  }
  for (int i = 0; i < 6; ++i) {
    p[i] = PyLong_AsVoidPtr(args[i]);
    if (PyErr_Occurred()) return nullptr;
  }
  f_rope_table = reinterpret_cast<decltype(f_rope_table)>(p[0]);
  f_qk_norm_rope = reinterpret_cast<decltype(f_qk_norm_rope)>(p[1]);
  f_quantize_rows = reinterpret_cast<decltype(f_quantize_rows)>(p[2]);
  f_linear_i8 = reinterpret_cast<decltype(f_linear_i8)>(p[3]);
  f_cache_store_q = reinterpret_cast<decltype(f_cache_store_q)>(p[4]);
  f_cache_apply_q = reinterpret_cast<decltype(f_cache_apply_q)>(p[5]);
  Py_RETURN_NONE;
}

#define ENTRY(name, f) {name, reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(f)), METH_FASTCALL, nullptr}
PyMethodDef methods[] = {ENTRY("init", init),
                         ENTRY("dc_rope_table", entry<rope_table>),
                         ENTRY("dc_qk_norm_rope", entry<qk_norm_rope>),
                         ENTRY("dc_quantize_rows", entry<quantize_rows>),
                         ENTRY("dc_linear_i8", entry<linear_i8>),
                         ENTRY("dc_cache_store_q", entry<cache_q<true>>),
                         ENTRY("dc_cache_apply_q", entry<cache_q<false>>),
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_binding", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__binding() { return PyModule_Create(&module); }

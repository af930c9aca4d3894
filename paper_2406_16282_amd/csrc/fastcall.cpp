// The common form of the binding's calls in native code: plain contiguous tensors on the
// current device, outputs allocated here, the current stream. A call of this form costs
// the host two or three microseconds beside its kernel launch, against six to eight for
// the same steps in Python (checks, allocations, argument conversion), which is what the
// smallest calls were bound by. Every function returns None for anything else (another
// type, device, layout or shape), and binding.py then takes its own path with its own
// errors; a status other than 0 comes back as an int.
//
// Nothing is kept between calls but the addresses of the library's functions and of
// torch's accessor of the current stream's raw handle.
#include <Python.h>

#include <ATen/core/Tensor.h>
#include <ATen/ops/empty.h>
#include <ATen/ops/empty_like.h>
#include <c10/core/impl/VirtualGuardImpl.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include <cmath>
#include <cstdint>

#include "lmbp.h"

namespace {

PyObject* g_raw_stream = nullptr;   // torch._C._cuda_getCurrentRawStream
enum { kFp32 = 0, kBf16 = 1 };

// A plain dense tensor in GPU memory with storage of its own type; no subclass.
bool plain(PyObject* o, at::Tensor& t) {
  if (!THPVariable_CheckExact(o)) return false;
  t = THPVariable_Unpack(o);
  return t.defined() && t.device().type() == c10::DeviceType::CUDA && t.layout() == c10::kStrided &&
         t.has_storage() && t.is_contiguous();
}
int dtype_of(const at::Tensor& t) {
  if (t.scalar_type() == at::kFloat) return kFp32;
  if (t.scalar_type() == at::kBFloat16) return kBf16;
  return -1;
}
bool on_current_device(const at::Tensor& t) {
  return c10::impl::VirtualGuardImpl(c10::DeviceType::CUDA).getDevice() == t.device();
}
bool same(const at::Tensor& a, const at::Tensor& b) {
  return a.scalar_type() == b.scalar_type() && a.numel() == b.numel() && a.device() == b.device();
}
// The current stream's raw handle; false with a Python error set.
bool stream_of(const at::Tensor& t, void*& s) {
  PyObject* index = PyLong_FromLong(t.device().index());
  if (index == nullptr) return false;
  PyObject* handle = PyObject_CallOneArg(g_raw_stream, index);
  Py_DECREF(index);
  if (handle == nullptr) return false;
  s = PyLong_AsVoidPtr(handle);
  Py_DECREF(handle);
  return !PyErr_Occurred();
}
at::Tensor words(int64_t count, const at::Tensor& like) {
  return at::empty({count}, like.options().dtype(at::kInt));
}
int64_t code_words(int64_t n) { return (n + 15) / 16; }

template <class... T>
PyObject* result(int status, const T&... t) {
  if (status != 0) return PyLong_FromLong(status);
  if constexpr (sizeof...(T) == 1) {
    return THPVariable_Wrap((t, ...));
  } else {
    PyObject* out = PyTuple_New(sizeof...(T));
    if (out == nullptr) return nullptr;
    Py_ssize_t i = 0;
    bool ok = true;
    auto add = [&](const at::Tensor& v) {
      PyObject* o = ok ? THPVariable_Wrap(v) : nullptr;
      if (o == nullptr) ok = false;
      else PyTuple_SET_ITEM(out, i++, o);
    };
    (add(t), ...);
    if (ok) return out;
    Py_DECREF(out);
    return nullptr;
  }
}

// Allocations and launches run without the interpreter's lock, as torch's and ctypes' do.
struct NoGil {
  PyThreadState* state = PyEval_SaveThread();
  ~NoGil() { PyEval_RestoreThread(state); }
};

template <class F>
F address(PyObject* o) {
  return reinterpret_cast<F>(PyLong_AsVoidPtr(o));
}

// (function, x) -> (y, codes)
PyObject* act_fwd(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  at::Tensor x;
  if (n != 2 || !plain(a[1], x)) Py_RETURN_NONE;
  const int dt = dtype_of(x);
  if (dt < 0 || !on_current_device(x)) Py_RETURN_NONE;
  void* s;
  if (!stream_of(x, s)) return nullptr;
  at::Tensor y, codes;
  const auto f = address<int (*)(int, int64_t, const void*, void*, void*, void*)>(a[0]);
  int status;
  {
    NoGil released;
    y = at::empty_like(x);
    codes = words(code_words(x.numel()), x);
    status = f(dt, x.numel(), x.data_ptr(), y.data_ptr(), codes.data_ptr(), s);
  }
  return result(status, y, codes);
  END_HANDLE_TH_ERRORS
}

// (function, dy, codes) -> dx
PyObject* act_bwd(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  at::Tensor dy, codes;
  if (n != 3 || !plain(a[1], dy) || !plain(a[2], codes)) Py_RETURN_NONE;
  const int dt = dtype_of(dy);
  if (dt < 0 || !on_current_device(dy) || codes.device() != dy.device() || codes.scalar_type() != at::kInt ||
      codes.numel() < code_words(dy.numel()))
    Py_RETURN_NONE;
  void* s;
  if (!stream_of(dy, s)) return nullptr;
  at::Tensor dx;
  const auto f = address<int (*)(int, int64_t, const void*, const void*, void*, void*)>(a[0]);
  int status;
  {
    NoGil released;
    dx = at::empty_like(dy);
    status = f(dt, dy.numel(), dy.data_ptr(), codes.data_ptr(), dx.data_ptr(), s);
  }
  return result(status, dx);
  END_HANDLE_TH_ERRORS
}

// (function, g, u) -> (h, s, codes)
PyObject* glu_fwd(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  at::Tensor g, u;
  if (n != 3 || !plain(a[1], g) || !plain(a[2], u)) Py_RETURN_NONE;
  const int dt = dtype_of(g);
  if (dt < 0 || !on_current_device(g) || !same(u, g)) Py_RETURN_NONE;
  void* st;
  if (!stream_of(g, st)) return nullptr;
  at::Tensor h, s, codes;
  const auto f = address<int (*)(int, int64_t, const void*, const void*, void*, void*, void*, void*)>(a[0]);
  int status;
  {
    NoGil released;
    h = at::empty_like(g);
    s = at::empty_like(g);
    codes = words(code_words(g.numel()), g);
    status = f(dt, g.numel(), g.data_ptr(), u.data_ptr(), h.data_ptr(), s.data_ptr(), codes.data_ptr(), st);
  }
  return result(status, h, s, codes);
  END_HANDLE_TH_ERRORS
}

// (function, dh, u, s, codes) -> (dg, du)
PyObject* glu_bwd(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  at::Tensor dh, u, s, codes;
  if (n != 5 || !plain(a[1], dh) || !plain(a[2], u) || !plain(a[3], s) || !plain(a[4], codes)) Py_RETURN_NONE;
  const int dt = dtype_of(dh);
  if (dt < 0 || !on_current_device(dh) || !same(u, dh) || !same(s, dh) || codes.device() != dh.device() ||
      codes.scalar_type() != at::kInt || codes.numel() < code_words(dh.numel()))
    Py_RETURN_NONE;
  void* st;
  if (!stream_of(dh, st)) return nullptr;
  at::Tensor dg, du;
  const auto f = address<int (*)(int, int64_t, const void*, const void*, const void*, const void*, void*, void*, void*)>(a[0]);
  int status;
  {
    NoGil released;
    dg = at::empty_like(dh);
    du = at::empty_like(dh);
    status = f(dt, dh.numel(), dh.data_ptr(), u.data_ptr(), s.data_ptr(), codes.data_ptr(), dg.data_ptr(),
               du.data_ptr(), st);
  }
  return result(status, dg, du);
  END_HANDLE_TH_ERRORS
}

// (function, x, eps) -> (z, rstd)
PyObject* norm_fwd(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  at::Tensor x;
  if (n != 3 || !PyFloat_CheckExact(a[2]) || !plain(a[1], x)) Py_RETURN_NONE;
  const int dt = dtype_of(x);
  if (dt < 0 || x.dim() == 0 || !on_current_device(x)) Py_RETURN_NONE;
  const int64_t cols = x.size(-1), rows = cols != 0 ? x.numel() / cols : 0;
  void* s;
  if (!stream_of(x, s)) return nullptr;
  at::Tensor z, rstd;
  const auto f = address<int (*)(int, int64_t, int64_t, float, const void*, void*, void*, void*)>(a[0]);
  int status;
  {
    NoGil released;
    z = at::empty_like(x);
    rstd = at::empty(x.sizes().slice(0, size_t(x.dim() - 1)), x.options().dtype(at::kFloat));
    status = f(dt, rows, cols, float(PyFloat_AS_DOUBLE(a[2])), x.data_ptr(), z.data_ptr(), rstd.data_ptr(), s);
  }
  return result(status, z, rstd);
  END_HANDLE_TH_ERRORS
}

// (function, dz, z, rstd) -> dx
PyObject* norm_bwd(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  at::Tensor dz, z, rstd;
  if (n != 4 || !plain(a[1], dz) || !plain(a[2], z) || !plain(a[3], rstd)) Py_RETURN_NONE;
  const int dt = dtype_of(dz);
  if (dt < 0 || dz.dim() == 0 || !on_current_device(dz) || !same(z, dz) || z.sizes() != dz.sizes()) Py_RETURN_NONE;
  const int64_t cols = dz.size(-1), rows = cols != 0 ? dz.numel() / cols : 0;
  if (rstd.device() != dz.device() || rstd.scalar_type() != at::kFloat || rstd.numel() != rows) Py_RETURN_NONE;
  void* s;
  if (!stream_of(dz, s)) return nullptr;
  at::Tensor dx;
  const auto f = address<int (*)(int, int64_t, int64_t, const void*, const void*, const void*, void*, void*)>(a[0]);
  int status;
  {
    NoGil released;
    dx = at::empty_like(dz);
    status = f(dt, rows, cols, dz.data_ptr(), z.data_ptr(), rstd.data_ptr(), dx.data_ptr(), s);
  }
  return result(status, dx);
  END_HANDLE_TH_ERRORS
}

// Sizes of a layer: x [.., k] and w [n, k], both bf16; false if they are anything else.
bool layer(const at::Tensor& x, const at::Tensor& w, int64_t& m, c10::SmallVector<int64_t, 6>& out) {
  if (x.scalar_type() != at::kBFloat16 || w.scalar_type() != at::kBFloat16 || w.dim() != 2 || x.dim() == 0 ||
      x.size(-1) != w.size(1) || w.device() != x.device() || !on_current_device(x))
    return false;
  out.assign(x.sizes().begin(), x.sizes().end());
  out.back() = w.size(0);
  m = 1;
  for (size_t i = 0; i + 1 < out.size(); ++i) m *= out[i];
  return true;
}

// (function, activation, x, w, bias or None) -> (y, codes)
PyObject* linear_act_fwd(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  at::Tensor x, w, b;
  int64_t m;
  c10::SmallVector<int64_t, 6> shape;
  if (n != 5 || !plain(a[2], x) || !plain(a[3], w) || !layer(x, w, m, shape)) Py_RETURN_NONE;
  if (a[4] != Py_None && (!plain(a[4], b) || b.scalar_type() != at::kBFloat16 || b.numel() != w.size(0) ||
                          b.device() != x.device()))
    Py_RETURN_NONE;
  void* s;
  if (!stream_of(x, s)) return nullptr;
  const int act = int(PyLong_AsLong(a[1]));
  at::Tensor y, codes;
  const auto f = address<int (*)(int, int, int64_t, int64_t, int64_t, const void*, const void*, const void*, void*,
                                 void*, void*, void*)>(a[0]);
  int status;
  {
    NoGil released;
    y = at::empty(shape, x.options());
    codes = words(code_words(m * w.size(0)), x);
    status = f(act, kBf16, m, w.size(0), w.size(1), x.data_ptr(), w.data_ptr(),
               b.defined() ? b.data_ptr() : nullptr, y.data_ptr(), codes.data_ptr(), nullptr, s);
  }
  return result(status, y, codes);
  END_HANDLE_TH_ERRORS
}

// (function, x, w_gate, w_up) -> (h, s, u, codes)
PyObject* linear_swiglu_fwd(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  at::Tensor x, wg, wu;
  int64_t m;
  c10::SmallVector<int64_t, 6> shape;
  if (n != 4 || !plain(a[1], x) || !plain(a[2], wg) || !plain(a[3], wu) || !layer(x, wg, m, shape) || !same(wu, wg) ||
      wu.sizes() != wg.sizes())
    Py_RETURN_NONE;
  void* st;
  if (!stream_of(x, st)) return nullptr;
  at::Tensor h, s, u, codes;
  const auto f = address<int (*)(int, int64_t, int64_t, int64_t, const void*, const void*, const void*, void*, void*,
                                 void*, void*, void*, void*)>(a[0]);
  int status;
  {
    NoGil released;
    h = at::empty(shape, x.options());
    s = at::empty(shape, x.options());
    u = at::empty(shape, x.options());
    codes = words(code_words(m * wg.size(0)), x);
    status = f(kBf16, m, wg.size(0), wg.size(1), x.data_ptr(), wg.data_ptr(), wu.data_ptr(), h.data_ptr(),
                s.data_ptr(), u.data_ptr(), codes.data_ptr(), nullptr, st);
  }
  return result(status, h, s, u, codes);
  END_HANDLE_TH_ERRORS
}

// (function, activation, x, w, eps, bias or None) -> (y, codes, z, rstd)
PyObject* norm_linear_act_fwd(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  at::Tensor x, w, b;
  int64_t m;
  c10::SmallVector<int64_t, 6> shape;
  if (n != 6 || !PyFloat_CheckExact(a[4]) || !plain(a[2], x) || !plain(a[3], w) || !layer(x, w, m, shape))
    Py_RETURN_NONE;
  if (a[5] != Py_None && (!plain(a[5], b) || b.scalar_type() != at::kBFloat16 || b.numel() != w.size(0) ||
                          b.device() != x.device()))
    Py_RETURN_NONE;
  void* s;
  if (!stream_of(x, s)) return nullptr;
  const int act = int(PyLong_AsLong(a[1]));
  at::Tensor y, codes, z, rstd;
  const auto f = address<int (*)(int, int, int64_t, int64_t, int64_t, float, const void*, const void*, const void*,
                                 void*, void*, void*, void*, void*, void*)>(a[0]);
  int status;
  {
    NoGil released;
    y = at::empty(shape, x.options());
    z = at::empty(x.sizes(), x.options());
    rstd = at::empty({m}, x.options().dtype(at::kFloat));
    codes = words(code_words(m * w.size(0)), x);
    status = f(act, kBf16, m, w.size(0), w.size(1), float(PyFloat_AS_DOUBLE(a[4])), x.data_ptr(), w.data_ptr(),
               b.defined() ? b.data_ptr() : nullptr, y.data_ptr(), codes.data_ptr(), nullptr, z.data_ptr(),
               rstd.data_ptr(), s);
  }
  return result(status, y, codes, z, rstd);
  END_HANDLE_TH_ERRORS
}

// (function, x, w_gate, w_up, eps) -> (h, s, u, codes, z, rstd)
PyObject* norm_linear_swiglu_fwd(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  at::Tensor x, wg, wu;
  int64_t m;
  c10::SmallVector<int64_t, 6> shape;
  if (n != 5 || !PyFloat_CheckExact(a[4]) || !plain(a[1], x) || !plain(a[2], wg) || !plain(a[3], wu) ||
      !layer(x, wg, m, shape) || !same(wu, wg) || wu.sizes() != wg.sizes())
    Py_RETURN_NONE;
  void* st;
  if (!stream_of(x, st)) return nullptr;
  at::Tensor h, s, u, codes, z, rstd;
  const auto f = address<int (*)(int, int64_t, int64_t, int64_t, float, const void*, const void*, const void*, void*,
                                 void*, void*, void*, void*, void*, void*, void*)>(a[0]);
  int status;
  {
    NoGil released;
    h = at::empty(shape, x.options());
    s = at::empty(shape, x.options());
    u = at::empty(shape, x.options());
    z = at::empty(x.sizes(), x.options());
    rstd = at::empty({m}, x.options().dtype(at::kFloat));
    codes = words(code_words(m * wg.size(0)), x);
    status = f(kBf16, m, wg.size(0), wg.size(1), float(PyFloat_AS_DOUBLE(a[4])), x.data_ptr(), wg.data_ptr(),
               wu.data_ptr(), h.data_ptr(), s.data_ptr(), u.data_ptr(), codes.data_ptr(), nullptr, z.data_ptr(),
               rstd.data_ptr(), st);
  }
  return result(status, h, s, u, codes, z, rstd);
  END_HANDLE_TH_ERRORS
}

// ---- rows and weights in 8 bits
bool f32_of(PyObject* o, const at::Tensor& like, int64_t count, at::Tensor& t) {
  return plain(o, t) && t.scalar_type() == at::kFloat && t.numel() == count && t.device() == like.device();
}
at::ScalarType type_of(int dt) { return dt == kBf16 ? at::kBFloat16 : at::kFloat; }
// Rows and columns of a tensor of at least one dimension; the sizes without the last one.
bool rows_of(const at::Tensor& t, int64_t& rows, int64_t& cols, at::IntArrayRef& lead) {
  if (t.dim() == 0) return false;
  cols = t.size(-1);
  lead = t.sizes().slice(0, size_t(t.dim() - 1));
  rows = 1;
  for (const int64_t v : lead) rows *= v;
  return true;
}

// (function, x) -> (q, scale)
PyObject* q8_rows(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  at::Tensor x;
  int64_t rows, cols;
  at::IntArrayRef lead;
  if (n != 2 || !plain(a[1], x) || !rows_of(x, rows, cols, lead)) Py_RETURN_NONE;
  const int dt = dtype_of(x);
  if (dt < 0 || !on_current_device(x)) Py_RETURN_NONE;
  void* s;
  if (!stream_of(x, s)) return nullptr;
  at::Tensor q, scale;
  const auto f = address<int (*)(int, int64_t, int64_t, const void*, void*, void*, void*)>(a[0]);
  int status;
  {
    NoGil released;
    q = at::empty(x.sizes(), x.options().dtype(at::kChar));
    scale = at::empty(lead, x.options().dtype(at::kFloat));
    status = f(dt, rows, cols, x.data_ptr(), q.data_ptr(), scale.data_ptr(), s);
  }
  return result(status, q, scale);
  END_HANDLE_TH_ERRORS
}

// (function, type, q, scale) -> v
PyObject* q8_values(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  at::Tensor q, scale;
  int64_t rows, cols;
  at::IntArrayRef lead;
  if (n != 4 || !plain(a[2], q) || q.scalar_type() != at::kChar || !rows_of(q, rows, cols, lead) || !on_current_device(q) ||
      !f32_of(a[3], q, rows, scale))
    Py_RETURN_NONE;
  const int dt = int(PyLong_AsLong(a[1]));
  void* s;
  if (!stream_of(q, s)) return nullptr;
  at::Tensor v;
  const auto f = address<int (*)(int, int64_t, int64_t, const void*, const void*, void*, void*)>(a[0]);
  int status;
  {
    NoGil released;
    v = at::empty(q.sizes(), q.options().dtype(type_of(dt)));
    status = f(dt, rows, cols, q.data_ptr(), scale.data_ptr(), v.data_ptr(), s);
  }
  return result(status, v);
  END_HANDLE_TH_ERRORS
}

// (function, x, eps, residual or None) -> (q, scale, rstd[, sum])
PyObject* msrms_q8_fwd(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  at::Tensor x, res;
  int64_t rows, cols;
  at::IntArrayRef lead;
  if (n != 4 || !PyFloat_CheckExact(a[2]) || !plain(a[1], x) || !rows_of(x, rows, cols, lead)) Py_RETURN_NONE;
  const int dt = dtype_of(x);
  if (dt < 0 || !on_current_device(x)) Py_RETURN_NONE;
  if (a[3] != Py_None && (!plain(a[3], res) || !same(res, x) || res.sizes() != x.sizes())) Py_RETURN_NONE;
  void* s;
  if (!stream_of(x, s)) return nullptr;
  at::Tensor q, scale, rstd, sum;
  const auto f = address<int (*)(int, int64_t, int64_t, float, const void*, const void*, void*, void*, void*, void*, void*)>(
      a[0]);
  int status;
  {
    NoGil released;
    q = at::empty(x.sizes(), x.options().dtype(at::kChar));
    scale = at::empty(lead, x.options().dtype(at::kFloat));
    rstd = at::empty(lead, x.options().dtype(at::kFloat));
    if (res.defined()) sum = at::empty(x.sizes(), x.options());
    status = f(dt, rows, cols, float(PyFloat_AS_DOUBLE(a[2])), x.data_ptr(), res.defined() ? res.data_ptr() : nullptr,
               sum.defined() ? sum.data_ptr() : nullptr, q.data_ptr(), scale.data_ptr(), rstd.data_ptr(), s);
  }
  return sum.defined() ? result(status, q, scale, rstd, sum) : result(status, q, scale, rstd);
  END_HANDLE_TH_ERRORS
}

// (function, type of dx, dz, q, scale, rstd, ds or None) -> dx
PyObject* msrms_q8_bwd(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  at::Tensor dz, q, scale, rstd, ds;
  int64_t rows, cols;
  at::IntArrayRef lead;
  if (n != 7 || !plain(a[2], dz) || !rows_of(dz, rows, cols, lead)) Py_RETURN_NONE;
  const int dt_dz = dtype_of(dz), dt = int(PyLong_AsLong(a[1]));
  if (dt_dz < 0 || !on_current_device(dz) || !plain(a[3], q) || q.scalar_type() != at::kChar || q.device() != dz.device() ||
      q.sizes() != dz.sizes() || !f32_of(a[4], dz, rows, scale) || !f32_of(a[5], dz, rows, rstd))
    Py_RETURN_NONE;
  if (a[6] != Py_None && (!plain(a[6], ds) || ds.scalar_type() != type_of(dt) || ds.device() != dz.device() ||
                          ds.sizes() != dz.sizes()))
    Py_RETURN_NONE;
  void* s;
  if (!stream_of(dz, s)) return nullptr;
  at::Tensor dx;
  const auto f = address<int (*)(int, int, int64_t, int64_t, const void*, const void*, const void*, const void*, const void*,
                                 void*, void*)>(a[0]);
  int status;
  {
    NoGil released;
    dx = at::empty(dz.sizes(), dz.options().dtype(type_of(dt)));
    status = f(dt_dz, dt, rows, cols, dz.data_ptr(), q.data_ptr(), scale.data_ptr(), rstd.data_ptr(),
               ds.defined() ? ds.data_ptr() : nullptr, dx.data_ptr(), s);
  }
  return result(status, dx);
  END_HANDLE_TH_ERRORS
}

// An 8-bit weight [n, k] and its scales on the device of `like`.
bool q8_weight(PyObject* ow, PyObject* os, const at::Tensor& like, at::Tensor& w, at::Tensor& w_scale) {
  return plain(ow, w) && w.scalar_type() == at::kChar && w.dim() == 2 && w.device() == like.device() &&
         f32_of(os, like, w.size(0), w_scale);
}

// (function, the workspace's size function, type, q, scale, w, w_scale, bias or None) -> y
PyObject* linear_q8_fwd(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  at::Tensor q, scale, w, w_scale, b;
  int64_t m, k;
  at::IntArrayRef lead;
  if (n != 8 || !plain(a[3], q) || q.scalar_type() != at::kChar || !rows_of(q, m, k, lead) || !on_current_device(q) ||
      !f32_of(a[4], q, m, scale) || !q8_weight(a[5], a[6], q, w, w_scale) || w.size(1) != k)
    Py_RETURN_NONE;
  const int dt = int(PyLong_AsLong(a[2]));
  if (a[7] != Py_None && (!plain(a[7], b) || b.scalar_type() != type_of(dt) || b.numel() != w.size(0) ||
                          b.device() != q.device()))
    Py_RETURN_NONE;
  void* s;
  if (!stream_of(q, s)) return nullptr;
  c10::SmallVector<int64_t, 6> shape(lead.begin(), lead.end());
  shape.push_back(w.size(0));
  at::Tensor y, work;
  const auto f = address<int (*)(int, int64_t, int64_t, int64_t, const void*, const void*, const void*, const void*,
                                 const void*, void*, void*, int64_t, void*)>(a[0]);
  const auto bytes_of = address<size_t (*)(int64_t, int64_t, int64_t)>(a[1]);
  int status;
  {
    NoGil released;
    const int64_t bytes = int64_t(bytes_of(m, w.size(0), k));
    if (bytes > 0) work = at::empty({bytes}, q.options().dtype(at::kByte));
    y = at::empty(shape, q.options().dtype(type_of(dt)));
    status = f(dt, m, w.size(0), k, q.data_ptr(), scale.data_ptr(), w.data_ptr(), w_scale.data_ptr(),
               b.defined() ? b.data_ptr() : nullptr, y.data_ptr(), bytes > 0 ? work.data_ptr() : nullptr, bytes, s);
  }
  return result(status, y);
  END_HANDLE_TH_ERRORS
}

// (function, the workspace's size function, type of dx, dy, w, w_scale, add or None, in place) -> dx
PyObject* linear_q8_bwd(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  at::Tensor dy, w, w_scale, add;
  int64_t m, cols;
  at::IntArrayRef lead;
  if (n != 8 || !plain(a[3], dy) || !rows_of(dy, m, cols, lead)) Py_RETURN_NONE;
  const int dt = dtype_of(dy), dt_dx = int(PyLong_AsLong(a[2]));
  if (dt < 0 || !on_current_device(dy) || !q8_weight(a[4], a[5], dy, w, w_scale) || w.size(0) != cols) Py_RETURN_NONE;
  void* s;
  if (!stream_of(dy, s)) return nullptr;
  c10::SmallVector<int64_t, 6> shape(lead.begin(), lead.end());
  shape.push_back(w.size(1));
  if (a[6] != Py_None && (!plain(a[6], add) || add.scalar_type() != type_of(dt_dx) || add.device() != dy.device() ||
                          add.sizes() != at::IntArrayRef(shape)))
    Py_RETURN_NONE;
  at::Tensor dx, work;
  const auto f = address<int (*)(int, int, int64_t, int64_t, int64_t, const void*, const void*, const void*, const void*,
                                 void*, void*, int64_t, void*)>(a[0]);
  const auto bytes_of = address<size_t (*)(int64_t, int64_t, int64_t)>(a[1]);
  int status;
  {
    NoGil released;
    const int64_t bytes = int64_t(bytes_of(m, cols, w.size(1)));
    work = at::empty({bytes}, dy.options().dtype(at::kByte));
    dx = a[7] == Py_True ? add : at::empty(shape, dy.options().dtype(type_of(dt_dx)));
    status = f(dt, dt_dx, m, cols, w.size(1), dy.data_ptr(), w.data_ptr(), w_scale.data_ptr(),
               add.defined() ? add.data_ptr() : nullptr, dx.data_ptr(), work.data_ptr(), bytes, s);
  }
  return result(status, dx);
  END_HANDLE_TH_ERRORS
}

// ---- tensors of heads

// A tensor in GPU memory, of any strides.
bool strided(PyObject* o, at::Tensor& t) {
  if (!THPVariable_CheckExact(o)) return false;
  t = THPVariable_Unpack(o);
  return t.defined() && t.device().type() == c10::DeviceType::CUDA && t.layout() == c10::kStrided && t.has_storage();
}
// The same, or None: an undefined tensor.
bool strided_or_none(PyObject* o, at::Tensor& t) { return o == Py_None || strided(o, t); }

// [.., heads, dim] with leading dimensions one behind the other, not empty.
struct Layout {
  int64_t rows, heads, dim;
  lmbp_heads view;
};
bool layout_of(const at::Tensor& t, Layout& l) {
  const int64_t n = t.dim();
  if (n < 3 || t.numel() == 0) return false;
  l.heads = t.size(n - 2);
  l.dim = t.size(n - 1);
  if (l.dim > 1 && t.stride(n - 1) != 1) return false;
  l.rows = 1;
  int64_t row = t.stride(n - 3), size = 0;
  for (int64_t i = n - 3; i >= 0; --i) {
    l.rows *= t.size(i);
    if (t.size(i) == 1) continue;
    if (size == 0) {
      row = t.stride(i);
      size = t.size(i);
    } else if (t.stride(i) != row * size) {
      return false;
    } else {
      size *= t.size(i);
    }
  }
  l.view.data = t.data_ptr();
  l.view.row = l.rows > 1 ? row : l.heads * l.dim;
  l.view.head = l.heads > 1 ? t.stride(n - 2) : l.dim;
  return true;
}
at::Tensor dense_like(const at::Tensor& t) { return at::empty(t.sizes(), t.options()); }
at::Tensor per_head(const at::Tensor& t) { return at::empty(t.sizes().slice(0, size_t(t.dim() - 1)), t.options().dtype(at::kFloat)); }
at::Tensor bytes_on(size_t count, const at::Tensor& t) { return at::empty({int64_t(count)}, t.options().dtype(at::kByte)); }
void* data_of(const at::Tensor& t) { return t.defined() ? t.data_ptr() : nullptr; }

// Queries and keys (k: or undefined) with positions and a rotation's address; false: anything but the common form.
bool rope_plan(const at::Tensor& q, const at::Tensor& k, PyObject* positions, PyObject* rotation, lmbp_rope& r, Layout& lq, Layout& lk) {
  if (dtype_of(q) < 0 || !on_current_device(q) || !layout_of(q, lq)) return false;
  if (k.defined() && (!layout_of(k, lk) || k.scalar_type() != q.scalar_type() || k.device() != q.device() || lk.rows != lq.rows ||
                      lk.dim != lq.dim))
    return false;
  r = *reinterpret_cast<const lmbp_rope*>(PyLong_AsVoidPtr(rotation));
  r.tokens = lq.rows;
  r.dim = lq.dim;
  r.q_heads = lq.heads;
  r.k_heads = k.defined() ? lk.heads : 0;
  if (2 * r.pairs > r.dim) return false;
  if (r.pairs > 0) {
    at::Tensor p;
    if (!plain(positions, p) || p.device() != q.device() || (p.scalar_type() != at::kLong && p.scalar_type() != at::kInt)) return false;
    const int64_t axes = p.numel() == lq.rows && r.n_axes == 1 ? 1 : p.dim() > 1 ? p.size(0) : 1;
    if (axes < r.n_axes || axes > 255 || p.numel() != axes * lq.rows) return false;
    r.n_axes = int(axes);
    r.wide = p.scalar_type() == at::kLong;
    r.positions = p.data_ptr();
  }
  return true;
}
// An output like t: the one given (None: allocated).
bool output(PyObject* o, const at::Tensor& like, at::Tensor& t, Layout& l) {
  if (o == Py_None) {
    t = dense_like(like);
  } else if (!strided(o, t) || t.scalar_type() != like.scalar_type() || t.device() != like.device() || t.sizes() != like.sizes()) {
    return false;
  }
  return layout_of(t, l);
}

// (function, q, k or None, positions, rotation, q_out or None, k_out or None) -> (q, k)
PyObject* rope(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  at::Tensor q, k, yq, yk;
  lmbp_rope r;
  Layout lq, lk, oq, ok;
  if (n != 7 || !strided(a[1], q) || !strided_or_none(a[2], k) || !rope_plan(q, k, a[3], a[4], r, lq, lk)) Py_RETURN_NONE;
  if (!output(a[5], q, yq, oq) || (k.defined() && !output(a[6], k, yk, ok))) Py_RETURN_NONE;
  void* s;
  if (!stream_of(q, s)) return nullptr;
  const auto f = address<decltype(&rope_fwd)>(a[0]);
  int status;
  {
    NoGil released;
    const bool two = k.defined();
    status = f(lmbp_dtype(dtype_of(q)), &r, &lq.view, two ? &lk.view : nullptr, &oq.view, two ? &ok.view : nullptr, s);
  }
  return result(status, yq, yk);
  END_HANDLE_TH_ERRORS
}

// Gains: both undefined, or one for each tensor, of one type.
bool gains_of(PyObject* oq, PyObject* ok, const at::Tensor& q, const at::Tensor& k, int64_t dim, at::Tensor& gq, at::Tensor& gk) {
  if ((oq != Py_None && !plain(oq, gq)) || (ok != Py_None && !plain(ok, gk))) return false;
  if (!gq.defined()) return !gk.defined();
  if (gk.defined() != k.defined() || dtype_of(gq) < 0 || gq.numel() != dim || gq.device() != q.device()) return false;
  return !gk.defined() || same(gk, gq);
}

// (function, q, k or None, eps, positions, rotation, q_gain, k_gain or None) -> (q, k, rstd_q, rstd_k)
PyObject* norm_rope_fwd(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  at::Tensor q, k, gq, gk, yq, yk, rq, rk;
  lmbp_rope r;
  Layout lq, lk, oq, ok;
  if (n != 8 || !strided(a[1], q) || !strided_or_none(a[2], k) || !PyFloat_CheckExact(a[3]) || !rope_plan(q, k, a[4], a[5], r, lq, lk) ||
      !gains_of(a[6], a[7], q, k, lq.dim, gq, gk))
    Py_RETURN_NONE;
  void* s;
  if (!stream_of(q, s)) return nullptr;
  const auto f = address<decltype(&msrms_rope_fwd)>(a[0]);
  const bool two = k.defined();
  int status;
  {
    NoGil released;
    yq = dense_like(q);
    rq = per_head(q);
    layout_of(yq, oq);
    if (two) {
      yk = dense_like(k);
      rk = per_head(k);
      layout_of(yk, ok);
    }
    status = f(lmbp_dtype(dtype_of(q)), lmbp_dtype(gq.defined() ? dtype_of(gq) : kBf16), &r, float(PyFloat_AS_DOUBLE(a[3])), data_of(gq),
               data_of(gk), &lq.view, two ? &lk.view : nullptr, &oq.view, two ? &ok.view : nullptr, rq.data_ptr<float>(),
               static_cast<float*>(data_of(rk)), s);
  }
  return result(status, yq, yk, rq, rk);
  END_HANDLE_TH_ERRORS
}

// (function, bytes, dq, dk or None, q, k, rstd_q, rstd_k, positions, rotation, q_gain, k_gain, q_out, k_out or None) ->
// (dq, dk) or (dq, dk, dq_gain, dk_gain)
PyObject* norm_rope_bwd(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  at::Tensor dq, dk, q, k, rq, rk, gq, gk, xq, xk, dgq, dgk, work;
  lmbp_rope r;
  Layout lq, lk, kq, kk, oq, ok;
  if (n != 14 || !strided(a[2], dq) || !strided_or_none(a[3], dk) || !strided(a[4], q) || !strided_or_none(a[5], k) || !plain(a[6], rq) ||
      !rope_plan(dq, dk, a[8], a[9], r, lq, lk) || !gains_of(a[10], a[11], dq, dk, lq.dim, gq, gk))
    Py_RETURN_NONE;
  const bool two = dk.defined();
  if (k.defined() != two || q.scalar_type() != dq.scalar_type() || q.device() != dq.device() || q.sizes() != dq.sizes() || !layout_of(q, kq) ||
      rq.device() != dq.device() || rq.scalar_type() != at::kFloat || rq.numel() != lq.rows * lq.heads)
    Py_RETURN_NONE;
  if (two && (k.scalar_type() != dq.scalar_type() || k.device() != dq.device() || k.sizes() != dk.sizes() || !layout_of(k, kk) ||
              !plain(a[7], rk) || rk.device() != dq.device() || rk.scalar_type() != at::kFloat || rk.numel() != lk.rows * lk.heads))
    Py_RETURN_NONE;
  if (!output(a[12], dq, xq, oq) || (two && !output(a[13], dk, xk, ok))) Py_RETURN_NONE;
  void* s;
  if (!stream_of(dq, s)) return nullptr;
  const auto f = address<decltype(&msrms_rope_bwd)>(a[0]);
  const auto bytes = address<decltype(&lmbp_msrms_rope_bwd_bytes)>(a[1]);
  int status;
  {
    NoGil released;
    size_t need = 0;
    if (gq.defined()) {
      need = bytes(lq.dim);
      work = bytes_on(need, dq);
      dgq = at::empty_like(gq);
      if (two) dgk = at::empty_like(gk);
    }
    status = f(lmbp_dtype(dtype_of(dq)), lmbp_dtype(gq.defined() ? dtype_of(gq) : kBf16), &r, data_of(gq), data_of(gk), &lq.view,
               two ? &lk.view : nullptr, &kq.view, two ? &kk.view : nullptr, rq.data_ptr<float>(), static_cast<const float*>(data_of(rk)),
               &oq.view, two ? &ok.view : nullptr, data_of(dgq), data_of(dgk), data_of(work), int64_t(need), s);
  }
  return gq.defined() ? result(status, xq, xk, dgq, dgk) : result(status, xq, xk);
  END_HANDLE_TH_ERRORS
}

// int32 numbers on q's device, or None.
bool numbers(PyObject* o, const at::Tensor& q, int64_t count, const int32_t*& p) {
  p = nullptr;
  if (o == Py_None) return true;
  at::Tensor t;
  if (!plain(o, t) || t.scalar_type() != at::kInt || t.device() != q.device() || t.numel() != count) return false;
  p = t.data_ptr<int32_t>();
  return true;
}
// Sequences of q or k; 0: not the common form.
int64_t sequences(const at::Tensor& t, PyObject* starts) {
  if (starts != Py_None) {
    at::Tensor s;
    return plain(starts, s) ? s.numel() - 1 : 0;
  }
  return t.dim() == 4 ? t.size(0) : t.dim() == 3 ? 1 : 0;
}
// a: q, k, v, causal, scale or None, q_starts, k_starts, k_lens.
bool attention_plan(PyObject* const* a, lmbp_attention& p, at::Tensor& q, at::Tensor& k, at::Tensor& v, Layout& lq, Layout& lk, Layout& lv) {
  if (!strided(a[0], q) || !strided(a[1], k) || !strided(a[2], v)) return false;
  for (const at::Tensor* t : {&q, &k, &v})
    if (t->scalar_type() != at::kBFloat16 || t->device() != q.device()) return false;
  if (!on_current_device(q) || !layout_of(q, lq) || !layout_of(k, lk) || !layout_of(v, lv) || k.sizes() != v.sizes() || lk.dim != lq.dim ||
      lq.heads % lk.heads != 0)
    return false;
  PyObject* k_starts = a[6];
  if (a[5] != Py_None && k_starts == Py_None && a[7] == Py_None && k.sizes().slice(0, size_t(k.dim() - 2)) == q.sizes().slice(0, size_t(q.dim() - 2)))
    k_starts = a[5];
  p.batch = sequences(q, a[5]);
  if (p.batch < 1 || sequences(k, k_starts) != p.batch) return false;
  if (!numbers(a[5], q, p.batch + 1, p.q_starts) || !numbers(k_starts, q, p.batch + 1, p.k_starts) || !numbers(a[7], q, p.batch, p.k_lens))
    return false;
  p.heads = lq.heads;
  p.kv_heads = lk.heads;
  p.dim = lq.dim;
  p.q_rows = lq.rows;
  p.k_rows = lk.rows;
  p.causal = a[3] == Py_True;
  if (a[3] != Py_True && a[3] != Py_False) return false;
  if (a[4] == Py_None) p.scale = float(1.0 / std::sqrt(double(lq.dim)));
  else if (PyFloat_CheckExact(a[4])) p.scale = float(PyFloat_AS_DOUBLE(a[4]));
  else return false;
  return true;
}

// (function, bytes, q, k, v, causal, scale, q_starts, k_starts, k_lens) -> (o, lse)
PyObject* attention_forward(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  at::Tensor q, k, v, o, lse, work;
  lmbp_attention p;
  Layout lq, lk, lv, lo;
  if (n != 10 || !attention_plan(a + 2, p, q, k, v, lq, lk, lv)) Py_RETURN_NONE;
  p.fill = 1;
  void* s;
  if (!stream_of(q, s)) return nullptr;
  const auto f = address<decltype(&attention_fwd)>(a[0]);
  const auto bytes = address<decltype(&lmbp_attention_fwd_bytes)>(a[1]);
  int status;
  {
    NoGil released;
    o = dense_like(q);
    lse = per_head(q);
    layout_of(o, lo);
    const size_t need = bytes(&p);
    if (need > 0) work = bytes_on(need, q);
    status = f(LMBP_BF16, &p, &lq.view, &lk.view, &lv.view, &lo.view, lse.data_ptr<float>(), data_of(work), int64_t(need), s);
  }
  return result(status, o, lse);
  END_HANDLE_TH_ERRORS
}

// (function, bytes, do, q, k, v, causal, scale, q_starts, k_starts, k_lens, o, lse, dq, dk, dv or None) -> (dq, dk, dv)
PyObject* attention_backward(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  at::Tensor d, q, k, v, o, lse, dq, dk, dv, work;
  lmbp_attention p;
  Layout ld, lq, lk, lv, lo, oq, ok, ov;
  if (n != 16 || !strided(a[2], d) || !attention_plan(a + 3, p, q, k, v, lq, lk, lv) || !strided(a[11], o) || !plain(a[12], lse)) Py_RETURN_NONE;
  for (const at::Tensor* t : {&d, &o})
    if (t->scalar_type() != at::kBFloat16 || t->device() != q.device() || t->sizes() != q.sizes()) Py_RETURN_NONE;
  if (!layout_of(d, ld) || !layout_of(o, lo) || lse.scalar_type() != at::kFloat || lse.device() != q.device() || lse.numel() != lq.rows * lq.heads)
    Py_RETURN_NONE;
  p.fill = a[13] == Py_None || a[14] == Py_None || a[15] == Py_None;
  if (!output(a[13], q, dq, oq) || !output(a[14], k, dk, ok) || !output(a[15], v, dv, ov)) Py_RETURN_NONE;
  void* s;
  if (!stream_of(q, s)) return nullptr;
  const auto f = address<decltype(&attention_bwd)>(a[0]);
  const auto bytes = address<decltype(&lmbp_attention_bwd_bytes)>(a[1]);
  int status;
  {
    NoGil released;
    const size_t need = bytes(&p);
    if (need > 0) work = bytes_on(need, q);
    status = f(LMBP_BF16, &p, &ld.view, &lq.view, &lk.view, &lv.view, &lo.view, lse.data_ptr<float>(), &oq.view, &ok.view, &ov.view,
               data_of(work), int64_t(need), s);
  }
  return result(status, dq, dk, dv);
  END_HANDLE_TH_ERRORS
}

// (torch's raw-stream accessor)
PyObject* bind(PyObject*, PyObject* accessor) {
  Py_INCREF(accessor);
  Py_XSETREF(g_raw_stream, accessor);
  Py_RETURN_NONE;
}

#define LMBP_FAST(name) {#name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(name)), METH_FASTCALL, nullptr}
PyMethodDef kMethods[] = {LMBP_FAST(act_fwd), LMBP_FAST(act_bwd), LMBP_FAST(glu_fwd), LMBP_FAST(glu_bwd),
                          LMBP_FAST(norm_fwd), LMBP_FAST(norm_bwd), LMBP_FAST(linear_act_fwd),
                          LMBP_FAST(linear_swiglu_fwd), LMBP_FAST(norm_linear_act_fwd),
                          LMBP_FAST(norm_linear_swiglu_fwd), LMBP_FAST(q8_rows), LMBP_FAST(q8_values),
                          LMBP_FAST(msrms_q8_fwd), LMBP_FAST(msrms_q8_bwd), LMBP_FAST(linear_q8_fwd),
                          LMBP_FAST(linear_q8_bwd), LMBP_FAST(rope), LMBP_FAST(norm_rope_fwd), LMBP_FAST(norm_rope_bwd),
                          LMBP_FAST(attention_forward), LMBP_FAST(attention_backward), {"bind", bind, METH_O, nullptr},
                          {nullptr, nullptr, 0, nullptr}};
PyModuleDef kModule = {PyModuleDef_HEAD_INIT, "_fastcall", nullptr, -1, kMethods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__fastcall() { return PyModule_Create(&kModule); }

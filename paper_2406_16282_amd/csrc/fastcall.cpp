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

#include <cstdint>

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
                          LMBP_FAST(linear_q8_bwd), {"bind", bind, METH_O, nullptr},
                          {nullptr, nullptr, 0, nullptr}};
PyModuleDef kModule = {PyModuleDef_HEAD_INIT, "_fastcall", nullptr, -1, kMethods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__fastcall() { return PyModule_Create(&kModule); }

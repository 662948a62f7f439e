// binding.cpp -- the Python calls of the operators around the attention
// (module _operators): checks tensors, fills the C ABI's argument structures
// and calls it.
//
// The other entry points are marshalled in Python (ctypes).  These are a few
// microseconds of GPU work at their smallest and take up to ten tensors of
// any strides each; checking those from Python took as long as the launch
// (3.4 of 7.0 us a call, against 0.4 here).
//
// Every function takes its arguments by position, None for an absent tensor,
// and a stream handle last (None: the current stream), and returns the call's
// status.
#include <Python.h>
#include <c10/hip/HIPStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include <string>

#include "dopr.h"

namespace {

using at::ScalarType;

struct Refused {};  // a Python error has been set

int32_t dtype_code(const at::Tensor &t, const char *what) {
  switch (t.scalar_type()) {
    case ScalarType::BFloat16: return DOPR_BF16;
    case ScalarType::Half: return DOPR_F16;
    case ScalarType::Float: return DOPR_F32;
    default: break;
  }
  PyErr_Format(PyExc_ValueError,
               "%s must be bfloat16, float16 or float32, not %s", what,
               toString(t.scalar_type()));
  throw Refused{};
}

std::string sizes(const int64_t *v, int64_t n) {
  std::string s = "(";
  for (int64_t i = 0; i < n; ++i)
    s += (i ? ", " : "") + std::to_string(v[i]);
  return s + ")";
}

const at::Tensor &tensor(PyObject *o, const char *what) {
  if (!THPVariable_Check(o)) {
    PyErr_Format(PyExc_ValueError, "%s must be a tensor", what);
    throw Refused{};
  }
  return THPVariable_Unpack(o);
}

// The tensor, if it is on a GPU and has this type, this shape and a unit last
// stride.
const at::Tensor &expect(PyObject *o, const char *what, ScalarType type,
                         std::initializer_list<int64_t> shape) {
  const at::Tensor &t = tensor(o, what);
  const int64_t dims = (int64_t)shape.size(), last = *(shape.end() - 1);
  bool good = t.scalar_type() == type && t.is_cuda() && t.dim() == dims;
  for (int64_t i = 0; good && i < dims; ++i)
    good = t.size(i) == shape.begin()[i];
  if (good && (last <= 1 || t.stride(-1) == 1)) return t;
  PyErr_Format(PyExc_ValueError,
               "%s must be a %s GPU tensor of shape %s with unit last stride, "
               "not %s %s, strides %s, on %s",
               what, toString(type), sizes(shape.begin(), dims).c_str(),
               toString(t.scalar_type()),
               sizes(t.sizes().data(), t.dim()).c_str(),
               sizes(t.strides().data(), t.dim()).c_str(),
               t.device().str().c_str());
  throw Refused{};
}

// A contiguous vector's address, NULL for None.
template <typename P>
void vector(PyObject *o, const char *what, ScalarType type, int64_t n, P &p) {
  p = o == Py_None ? nullptr
                   : static_cast<P>(expect(o, what, type, {n}).data_ptr());
}

// A matrix's address and row stride, NULL and 0 for None; a single row has no
// stride to speak of.
template <typename P>
void matrix(PyObject *o, const char *what, ScalarType type, int64_t rows,
            int64_t width, P &p, int64_t &stride) {
  p = nullptr;
  stride = 0;
  if (o == Py_None) return;
  const at::Tensor &t = expect(o, what, type, {rows, width});
  p = static_cast<P>(t.data_ptr());
  stride = rows > 1 ? t.stride(0) : std::max(t.stride(0), width);
}

void two_dims(const at::Tensor &t, const char *what) {
  if (t.dim() == 2) return;
  PyErr_Format(PyExc_ValueError, "%s must have two dimensions, not %d", what,
               (int)t.dim());
  throw Refused{};
}

// The stream's handle; None is the current device's current stream.
void *handle(PyObject *o) {
  if (o == Py_None) return c10::hip::getCurrentHIPStream().stream();
  void *p = PyLong_AsVoidPtr(o);
  if (!p && PyErr_Occurred()) throw Refused{};
  return p;
}

float real(PyObject *o) {
  const double v = PyFloat_AsDouble(o);
  if (v == -1.0 && PyErr_Occurred()) throw Refused{};
  return (float)v;
}

int32_t flag(PyObject *o) {
  const int v = PyObject_IsTrue(o);
  if (v < 0) throw Refused{};  // (an error of the object's own)
  return v;
}

PyObject *quantize_rows(PyObject *const *a) {
  dopr_quantize_args_t s{};
  const at::Tensor &x = tensor(a[0], "x");
  two_dims(x, "x");
  s.dtype = dtype_code(x, "x");
  s.rows = x.size(0);
  s.width = x.size(1);
  const ScalarType t = x.scalar_type();
  matrix(a[0], "x", t, s.rows, s.width, s.x, s.x_row_stride);
  matrix(a[1], "q", ScalarType::Char, s.rows, s.width, s.q, s.q_row_stride);
  vector(a[2], "scale", ScalarType::Float, s.rows, s.scale);
  matrix(a[3], "up", t, s.rows, s.width, s.up, s.up_row_stride);
  return PyLong_FromLong(dopr_quantize_rows(&s, handle(a[4])));
}

PyObject *quant_matmul(PyObject *const *a) {
  dopr_quant_matmul_args_t s{};
  const at::Tensor &x = tensor(a[0], "x"), &w = tensor(a[2], "w");
  const at::Tensor &y = tensor(a[4], "y");
  two_dims(x, "x");
  two_dims(w, "w");
  s.dtype = dtype_code(y, "y");
  s.rows = x.size(0);
  s.depth = x.size(1);
  s.cols = w.size(0);
  const ScalarType t = y.scalar_type(), i8 = ScalarType::Char;
  matrix(a[0], "x", i8, s.rows, s.depth, s.x, s.x_row_stride);
  vector(a[1], "x_scale", ScalarType::Float, s.rows, s.x_scale);
  matrix(a[2], "w", i8, s.cols, s.depth, s.w, s.w_row_stride);
  vector(a[3], "w_scale", ScalarType::Float, s.cols, s.w_scale);
  matrix(a[4], "y", t, s.rows, s.cols, s.y, s.y_row_stride);
  vector(a[5], "bias", t, s.cols, s.bias);
  matrix(a[6], "residual", t, s.rows, s.cols, s.residual,
         s.residual_row_stride);
  if (a[7] != Py_None) {
    const at::Tensor &ws = tensor(a[7], "workspace");
    if (!ws.is_cuda() || !ws.is_contiguous()) {
      PyErr_SetString(PyExc_ValueError,
                      "workspace must be a contiguous GPU tensor");
      throw Refused{};
    }
    s.workspace = ws.data_ptr();
    s.workspace_bytes = ws.nbytes();
  }
  return PyLong_FromLong(dopr_quant_matmul(&s, handle(a[8])));
}

PyObject *norm_residual(PyObject *const *a) {
  // x, residual, post_norm_w, gate, residual_scale, pre_norm_w, h, z, q,
  // q_scale, rms_eps, stream
  dopr_norm_residual_args_t s{};
  const at::Tensor &x = tensor(a[0], "x");
  two_dims(x, "x");
  s.dtype = s.residual_dtype = dtype_code(x, "x");
  s.rows = x.size(0);
  s.width = x.size(1);
  const ScalarType t = x.scalar_type();
  // residual and h: x's type, or fp32 kept wider than it
  PyObject *kept = a[1] != Py_None ? a[1] : a[6];
  ScalarType rt = t;
  if (kept != Py_None &&
      tensor(kept, "residual and h").scalar_type() == ScalarType::Float) {
    rt = ScalarType::Float;
    s.residual_dtype = DOPR_F32;
  }
  matrix(a[0], "x", t, s.rows, s.width, s.x, s.x_row_stride);
  matrix(a[1], "residual", rt, s.rows, s.width, s.residual,
         s.residual_row_stride);
  vector(a[2], "post_norm_w", t, s.width, s.post_norm_w);
  if (a[3] != Py_None && tensor(a[3], "gate").dim() == 1)
    vector(a[3], "gate", t, s.width, s.gate);
  else
    matrix(a[3], "gate", t, s.rows, s.width, s.gate, s.gate_row_stride);
  s.residual_scale = real(a[4]);
  vector(a[5], "pre_norm_w", t, s.width, s.pre_norm_w);
  matrix(a[6], "h", rt, s.rows, s.width, s.h, s.h_row_stride);
  matrix(a[7], "z", t, s.rows, s.width, s.z, s.z_row_stride);
  matrix(a[8], "q", ScalarType::Char, s.rows, s.width, s.q, s.q_row_stride);
  vector(a[9], "q_scale", ScalarType::Float, s.rows, s.q_scale);
  s.rms_eps = real(a[10]);
  return PyLong_FromLong(dopr_norm_residual(&s, handle(a[11])));
}

// [rows, heads, d] and its output
template <typename P>
void heads(PyObject *x, PyObject *out, const char *what, const char *out_what,
           ScalarType type, int64_t rows, int64_t d, int32_t &n, P &p,
           int64_t &row, int64_t &head, void *&o, int64_t &o_row,
           int64_t &o_head) {
  if (x == Py_None) return;
  const at::Tensor &t = tensor(x, what);
  const int64_t h = t.dim() == 3 ? t.size(1) : -1;
  expect(x, what, type, {rows, h, d});
  const at::Tensor &u = expect(out, out_what, type, {rows, h, d});
  if (h > INT32_MAX || d > INT32_MAX) {
    PyErr_Format(PyExc_ValueError, "%s has too many heads or elements", what);
    throw Refused{};
  }
  n = (int32_t)h;
  p = t.data_ptr();
  row = t.stride(0);
  head = t.stride(1);
  o = u.data_ptr();
  o_row = u.stride(0);
  o_head = u.stride(1);
}

PyObject *rotary(PyObject *const *a) {
  // q, k, positions, inv_freq, q_out, k_out, interleaved, inverse,
  // attention_factor, q_norm_w, k_norm_w, rms_eps, stream
  dopr_rotary_args_t s{};
  s.interleaved = flag(a[6]);
  s.inverse = flag(a[7]);
  if (a[0] == Py_None && a[1] == Py_None) {
    PyErr_SetString(PyExc_ValueError, "q and k are both None");
    throw Refused{};
  }
  const char *name = a[0] != Py_None ? "q" : "k";
  const at::Tensor &x = tensor(a[0] != Py_None ? a[0] : a[1], name);
  if (x.dim() != 3) {
    PyErr_Format(PyExc_ValueError, "%s must be [rows, heads, head_dim]", name);
    throw Refused{};
  }
  const ScalarType t = x.scalar_type();
  s.dtype = dtype_code(x, name);
  s.rows = x.size(0);
  s.head_dim = (int32_t)x.size(2);
  heads(a[0], a[4], "q", "q_out", t, s.rows, s.head_dim, s.n_q_heads, s.q,
        s.q_row_stride, s.q_head_stride, s.q_out, s.q_out_row_stride,
        s.q_out_head_stride);
  heads(a[1], a[5], "k", "k_out", t, s.rows, s.head_dim, s.n_kv_heads, s.k,
        s.k_row_stride, s.k_head_stride, s.k_out, s.k_out_row_stride,
        s.k_out_head_stride);
  vector(a[2], "positions", ScalarType::Int, s.rows, s.positions);
  const int64_t half = tensor(a[3], "inv_freq").numel();
  vector(a[3], "inv_freq", ScalarType::Float, half, s.inv_freq);
  s.rotary_dim = (int32_t)(2 * half);
  s.attention_factor = real(a[8]);
  vector(a[9], "q_norm_w", t, s.head_dim, s.q_norm_w);
  vector(a[10], "k_norm_w", t, s.head_dim, s.k_norm_w);
  s.rms_eps = real(a[11]);
  return PyLong_FromLong(dopr_rotary(&s, handle(a[12])));
}

template <PyObject *(*call)(PyObject *const *), Py_ssize_t count>
PyObject *entry(PyObject *, PyObject *const *args, Py_ssize_t n) {
  if (n != count) {
    PyErr_Format(PyExc_TypeError, "expected %zd arguments, got %zd", count, n);
    return nullptr;
  }
  try {
    return call(args);
  } catch (const Refused &) {
  } catch (const std::exception &e) {
    PyErr_SetString(PyExc_RuntimeError, e.what());
  }
  return nullptr;
}

#define DOPR_ENTRY(name, count)                                               \
  {#name, (PyCFunction)(void (*)(void))entry<name, count>, METH_FASTCALL,     \
   nullptr}

PyMethodDef methods[] = {DOPR_ENTRY(quantize_rows, 5),
                         DOPR_ENTRY(quant_matmul, 9),
                         DOPR_ENTRY(norm_residual, 12),
                         DOPR_ENTRY(rotary, 13),
                         {nullptr, nullptr, 0, nullptr}};

PyModuleDef module = {PyModuleDef_HEAD_INIT,
                      "_operators",
                      "Calls of the operators around the attention.",
                      -1,
                      methods,
                      nullptr,
                      nullptr,
                      nullptr,
                      nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__operators(void) { return PyModule_Create(&module); }

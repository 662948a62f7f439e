// binding.cpp -- the Python calls of the operators around the attention, of
// dopr_store_put_rotary, dopr_prefix_attn and dopr_gather_prefix (module
// _operators): checks tensors, fills the C ABI's argument structures and calls
// it.
//
// The other entry points are marshalled in Python (ctypes).  These are a few
// microseconds of GPU work at their smallest and take up to ten tensors of
// any strides each; checking those from Python took as long as the launch
// (3.4 of 7.0 us a call, against 0.4 here).
//
// Every function takes its arguments by position, None for an absent tensor,
// and a stream handle last (None: the current stream), and returns the call's
// status, or None where it has not been made (see Elsewhere).
#include <Python.h>
#include <c10/hip/HIPStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include <cmath>
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

// The status of a C call, which other Python threads run beside: it waits where
// the stream's queue is full.
template <typename Call>
PyObject *status_of(Call call) {
  struct Unlocked {
    PyThreadState *state = PyEval_SaveThread();
    ~Unlocked() { PyEval_RestoreThread(state); }
  };
  const auto made = [&] {
    const Unlocked here;
    return call();
  };
  return PyLong_FromLong(made());
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
  void *stream = handle(a[4]);
  return status_of([&] { return dopr_quantize_rows(&s, stream); });
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
  void *stream = handle(a[8]);
  return status_of([&] { return dopr_quant_matmul(&s, stream); });
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
  void *stream = handle(a[11]);
  return status_of([&] { return dopr_norm_residual(&s, stream); });
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
  void *stream = handle(a[12]);
  return status_of([&] { return dopr_rotary(&s, stream); });
}

int64_t whole(PyObject *o) {
  const long long v = PyLong_AsLongLong(o);
  if (v == -1 && PyErr_Occurred()) throw Refused{};
  return v;
}

PyObject *store_put_rotary(PyObject *const *a) {
  // store's handle, kv heads, head dim and device, layer, doc_ids,
  // src_cu_slots, k, v, inv_freq, positions, k_norm_w, interleaved,
  // attention_factor, rms_eps, stream
  dopr_put_rotary_args_t s{};
  const int64_t hkv = whole(a[1]), d = whole(a[2]), device = whole(a[3]);
  const int64_t layer = whole(a[4]);
  s.layer = (int32_t)std::max<int64_t>(-1, std::min<int64_t>(layer,
                                                             INT32_MAX));
  const at::Tensor &k = tensor(a[7], "k");
  if (k.dim() != 3) {
    PyErr_SetString(PyExc_ValueError, "k must be [rows, kv heads, head dim]");
    throw Refused{};
  }
  s.dtype = dtype_code(k, "k");
  s.rows = k.size(0);
  const ScalarType t = k.scalar_type();
  expect(a[7], "k", t, {s.rows, hkv, d});
  const at::Tensor &v = expect(a[8], "v", t, {s.rows, hkv, d});
  s.k = k.data_ptr();
  s.k_row_stride = k.stride(0);
  s.k_head_stride = k.stride(1);
  s.v = v.data_ptr();
  s.v_row_stride = v.stride(0);
  s.v_head_stride = v.stride(1);
  s.n = tensor(a[5], "doc_ids").numel();
  vector(a[5], "doc_ids", ScalarType::Int, s.n, s.doc_ids);
  vector(a[6], "src_cu_slots", ScalarType::Long, s.n + 1, s.src_cu_slots);
  const int64_t half = tensor(a[9], "inv_freq").numel();
  vector(a[9], "inv_freq", ScalarType::Float, half, s.inv_freq);
  s.rotary_dim = (int32_t)std::min<int64_t>(2 * half, INT32_MAX - 1);
  vector(a[10], "positions", ScalarType::Int, s.rows, s.positions);
  vector(a[11], "k_norm_w", t, d, s.k_norm_w);
  const char *names[] = {"doc_ids", "src_cu_slots", "k",        "v",
                         "inv_freq", "positions",    "k_norm_w"};
  for (int i = 0; i < 7; ++i)
    if (a[5 + i] != Py_None && tensor(a[5 + i], names[i]).device().index() !=
                                   device) {
      PyErr_Format(PyExc_ValueError, "%s must be on the store's device",
                   names[i]);
      throw Refused{};
    }
  s.interleaved = flag(a[12]);
  s.attention_factor = real(a[13]);
  s.rms_eps = real(a[14]);
  void *store = PyLong_AsVoidPtr(a[0]);
  if (!store && PyErr_Occurred()) throw Refused{};
  void *stream = handle(a[15]);
  return status_of([&] {
    return dopr_store_put_rotary(static_cast<dopr_store_t>(store), &s, stream);
  });
}

// The calls below are also marshalled in Python, which takes more than they do
// (other objects with a tensor's methods, numbers and handles in other forms) and
// names what it refuses; an argument of another kind than a tensor, an int or a
// float leaves the call to that.
struct Elsewhere {};

// A tensor's address as it is (its caller keeps to the C ABI), NULL for None.
template <typename P>
void address(PyObject *o, P &p) {
  if (o != Py_None && !THPVariable_Check(o)) throw Elsewhere{};
  p = o == Py_None ? nullptr
                   : static_cast<P>(THPVariable_Unpack(o).data_ptr());
}

const at::Tensor &plain_tensor(PyObject *o) {
  if (!THPVariable_Check(o)) throw Elsewhere{};
  return THPVariable_Unpack(o);
}

// An int's lowest bits as the C type (as ctypes passes it), a handle's with None
// for NULL.
template <typename I>
I bits(PyObject *o) {
  if (!PyLong_Check(o)) throw Elsewhere{};
  const unsigned long long v = PyLong_AsUnsignedLongLongMask(o);
  if (v == ~0ull && PyErr_Occurred()) throw Refused{};
  return (I)v;
}

void *pointer(PyObject *o) {
  return o == Py_None ? nullptr : reinterpret_cast<void *>(bits<uintptr_t>(o));
}

float plain_real(PyObject *o) {
  if (!PyFloat_Check(o) && !PyLong_Check(o)) throw Elsewhere{};
  return real(o);
}

void *plain_handle(PyObject *o) {
  return o == Py_None ? handle(o) : pointer(o);
}

PyObject *prefix_attn(PyObject *const *a) {
  // store's handle, kv heads and head dim, layer, doc_ids, cu_seqlens, q, k, v,
  // q_norm_w, k_norm_w, out, lse, workspace, max_tokens, total_tokens, rms_eps,
  // rope_theta, softmax_scale, kernel_variant, timing begin and end,
  // rope_inv_freq, rows_per_item, queue_order, stream
  dopr_attn_args_t s{};
  s.n_pairs = (int32_t)plain_tensor(a[4]).numel();
  address(a[4], s.doc_ids);
  address(a[5], s.cu_seqlens);
  s.n_q_heads = bits<int32_t>(a[1]);
  if (a[6] != Py_None) {
    const at::Tensor &q = plain_tensor(a[6]);
    if (q.dim() < 2) throw Elsewhere{};
    s.n_q_heads = (int32_t)q.size(1);
    s.total_tokens = q.size(0);
  } else if (a[15] == Py_None) {
    throw Elsewhere{};
  }
  address(a[6], s.q);
  address(a[7], s.k);
  address(a[8], s.v);
  address(a[9], s.q_norm_w);
  address(a[10], s.k_norm_w);
  address(a[11], s.out);
  address(a[12], s.lse);
  address(a[13], s.workspace);
  if (s.workspace) s.workspace_bytes = plain_tensor(a[13]).nbytes();
  s.max_tokens = bits<int32_t>(a[14]);
  if (a[15] != Py_None) s.total_tokens = bits<int64_t>(a[15]);
  s.rms_eps = plain_real(a[16]);
  s.rope_theta = plain_real(a[17]);
  s.softmax_scale =
      a[18] == Py_None
          ? (float)std::pow((double)bits<int32_t>(a[2]), -0.5)
          : plain_real(a[18]);
  s.kernel_variant = bits<int32_t>(a[19]);
  s.timing_begin = pointer(a[20]);
  s.timing_end = pointer(a[21]);
  address(a[22], s.rope_inv_freq);
  s.rows_per_item = bits<int32_t>(a[23]);
  s.queue_order = bits<int32_t>(a[24]);
  const auto store = static_cast<dopr_store_t>(pointer(a[0]));
  const int32_t layer = bits<int32_t>(a[3]);
  void *stream = plain_handle(a[25]);
  return status_of([&] { return dopr_prefix_attn(store, layer, &s, stream); });
}

PyObject *gather_prefix(PyObject *const *a) {
  // store's handle, layer, doc_ids, out_cu_slots, k_out, v_out, stream
  const int32_t *doc_ids;
  const int64_t *out_cu;
  void *k, *v;
  address(a[2], doc_ids);
  address(a[3], out_cu);
  address(a[4], k);
  address(a[5], v);
  const auto store = static_cast<dopr_store_t>(pointer(a[0]));
  const int32_t layer = bits<int32_t>(a[1]);
  const int32_t n = (int32_t)plain_tensor(a[2]).numel();
  void *stream = plain_handle(a[6]);
  return status_of([&] {
    return dopr_gather_prefix(store, layer, n, doc_ids, out_cu, k, v, stream);
  });
}

template <PyObject *(*call)(PyObject *const *), Py_ssize_t count>
PyObject *entry(PyObject *, PyObject *const *args, Py_ssize_t n) {
  if (n != count) {
    PyErr_Format(PyExc_TypeError, "expected %zd arguments, got %zd", count, n);
    return nullptr;
  }
  try {
    return call(args);
  } catch (const Elsewhere &) {
    Py_RETURN_NONE;
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
                         DOPR_ENTRY(store_put_rotary, 16),
                         DOPR_ENTRY(prefix_attn, 26),
                         DOPR_ENTRY(gather_prefix, 7),
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

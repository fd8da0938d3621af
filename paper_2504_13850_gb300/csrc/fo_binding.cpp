// Python binding of the embedding, norm and orthogonalisation entry points on
// torch tensors (argument marshalling only; api.py has the documentation).
//
// These calls are short: through ctypes, with the checks and allocations in
// Python, they took 10 to 20 us of host time, several times what their kernels
// take on a batch of 4096 x 512.  Here the checks read the tensors' fields and
// outputs come straight from torch's allocator.
#include <Python.h>

#include <ATen/core/TensorBase.h>
#include <ATen/cuda/EmptyTensor.h>
#include <c10/cuda/CUDAGuard.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/Dtype.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>
#include <torch/csrc/utils/object_ptr.h>

#include <cstdarg>
#include <optional>
#include <vector>

#include "../../include/fedoptima.h"

namespace {

using at::ScalarType;
using at::TensorBase;

PyObject* g_error = nullptr;      // api.FedOptimaError

[[noreturn]] void refuse(PyObject* kind, const char* format, ...) {
  va_list args;
  va_start(args, format);
  PyErr_FormatV(kind, format, args);
  va_end(args);
  throw python_error();
}

void check(int rc, const char* what) {
  if (rc >= 0) return;
  static const char* const names[] = {"ERR_ARG", "ERR_CUDA", "ERR_OOM", "ERR_TIMEOUT", "ERR_UNSUPPORTED"};
  refuse(g_error ? g_error : PyExc_RuntimeError, "%s: %s: %s", what, rc >= -5 ? names[-rc - 1] : "error", fo_last_error());
}

const at::Tensor& tensor(PyObject* o, const char* name) {
  if (!THPVariable_Check(o)) refuse(PyExc_TypeError, "%s: a tensor is wanted", name);
  return THPVariable_Unpack(o);
}
int64_t integer(PyObject* o) {
  const int64_t v = PyLong_AsLongLong(o);
  if (v == -1 && PyErr_Occurred()) throw python_error();
  return v;
}
double real(PyObject* o) {
  const double v = PyFloat_AsDouble(o);
  if (v == -1.0 && PyErr_Occurred()) throw python_error();
  return v;
}
bool truth(PyObject* o) {
  const int v = PyObject_IsTrue(o);
  if (v < 0) throw python_error();
  return v != 0;
}
int code(const TensorBase& t, const char* name) {
  if (t.scalar_type() == ScalarType::BFloat16) return FO_DTYPE_BF16;
  if (t.scalar_type() == ScalarType::Float) return FO_DTYPE_F32;
  refuse(PyExc_ValueError, "%s: bf16 or fp32", name);
}
// A Python dtype, or `other` for None.
ScalarType dtype_of(PyObject* o, ScalarType other) {
  if (o == Py_None) return other;
  if (!THPDtype_Check(o)) refuse(PyExc_TypeError, "dtype: a torch dtype is wanted");
  return reinterpret_cast<THPDtype*>(o)->scalar_type;
}

struct Rows {
  void* data = nullptr;
  int64_t stride = 0;
};
// `t` seen as a matrix [rows, last dimension]: contiguous, or two dimensions with
// innermost stride 1.
Rows rows_of(const TensorBase& t, at::IntArrayRef shape, ScalarType type, int device, const char* name) {
  if (t.sizes() != shape || t.scalar_type() != type || t.get_device() != device)
    refuse(PyExc_ValueError, "%s: the shape, type and device of the others are wanted", name);
  if (t.is_contiguous()) return {t.data_ptr(), shape.back()};
  if (shape.size() == 2 && t.stride(1) == 1) return {t.data_ptr(), t.stride(0)};
  refuse(PyExc_ValueError, "%s: contiguous, or a matrix with innermost stride 1", name);
}
void* small(const TensorBase& t, at::IntArrayRef shape, ScalarType type, int device, const char* name) {
  if (t.sizes() != shape || t.scalar_type() != type || t.get_device() != device || !t.is_contiguous())
    refuse(PyExc_ValueError, "%s: a contiguous tensor of the right shape and type on the others' device", name);
  return t.data_ptr();
}
// `o`, or a contiguous copy where its strides would refuse it: autograd hands over
// gradients broadcast by a sum or a mean.
struct Dense {
  THPObjectPtr copy;
  const at::Tensor* t;
  Dense(PyObject* o, const char* name) : t(&tensor(o, name)) {
    if (t->is_contiguous() || (t->dim() == 2 && t->stride(1) == 1)) return;
    copy = THPObjectPtr(PyObject_CallMethod(o, "contiguous", nullptr));
    if (!copy) throw python_error();
    t = &THPVariable_Unpack(copy.get());
  }
  const at::Tensor* operator->() const { return t; }
  const at::Tensor& operator*() const { return *t; }
};

// The tensors' device is current and what a call allocates belongs to its stream.
struct Place {
  std::optional<c10::cuda::CUDAGuard> device;
  std::optional<c10::cuda::CUDAStreamGuard> guard;
  cudaStream_t stream;
  int index;
  Place(const TensorBase& t, PyObject* wanted) : index(t.get_device()) {
    if (!t.is_cuda()) refuse(PyExc_ValueError, "device tensors are wanted");
    if (index != c10::cuda::current_device()) device.emplace(c10::DeviceIndex(index));
    if (wanted == Py_None) {
      stream = c10::cuda::getCurrentCUDAStream(c10::DeviceIndex(index)).stream();
    } else {
      stream = reinterpret_cast<cudaStream_t>(static_cast<uintptr_t>(integer(wanted)));
      guard.emplace(c10::cuda::getStreamFromExternal(stream, c10::DeviceIndex(index)));
    }
  }
  at::Tensor empty(at::IntArrayRef shape, ScalarType type) const {
    return at::Tensor(at::detail::empty_cuda(shape, type, c10::Device(c10::kCUDA, c10::DeviceIndex(index)), std::nullopt));
  }
};

PyObject* tuple(std::initializer_list<const at::Tensor*> items) {
  THPObjectPtr r(PyTuple_New(Py_ssize_t(items.size())));
  if (!r) throw python_error();
  Py_ssize_t i = 0;
  for (const at::Tensor* t : items) {
    PyObject* o = THPVariable_Wrap(*t);
    if (!o) throw python_error();
    PyTuple_SET_ITEM(r.get(), i++, o);
  }
  return r.release();
}
void count(Py_ssize_t n, Py_ssize_t want) {
  if (n != want) refuse(PyExc_TypeError, "%d arguments are wanted", int(want));
}

std::pair<void*, int> ids_of(const TensorBase& ids) {
  const ScalarType t = ids.scalar_type();
  if (t != ScalarType::Int && t != ScalarType::Long) refuse(PyExc_ValueError, "ids: int32 or int64");
  if (!ids.is_contiguous()) refuse(PyExc_ValueError, "ids: contiguous");
  return {ids.data_ptr(), t == ScalarType::Int ? 32 : 64};
}
at::DimVector with_width(const TensorBase& ids, int64_t width) {
  at::DimVector shape(ids.sizes().begin(), ids.sizes().end());
  shape.push_back(width);
  return shape;
}

// embedding(ids, table, scale, dtype, out, stream)
PyObject* embedding(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  count(n, 6);
  const at::Tensor &ids = tensor(a[0], "ids"), &table = tensor(a[1], "table");
  const Place at(ids, a[5]);
  const auto [ip, bits] = ids_of(ids);
  if (table.dim() != 2 || !table.is_contiguous() || table.get_device() != at.index)
    refuse(PyExc_ValueError, "table: a contiguous matrix [vocab, width] on the ids' device");
  const int64_t width = table.size(1);
  const at::DimVector shape = with_width(ids, width);
  const ScalarType type = dtype_of(a[3], table.scalar_type());
  const at::Tensor out = a[4] == Py_None ? at.empty(shape, type) : tensor(a[4], "out");
  const Rows y = rows_of(out, shape, type, at.index, "out");
  check(fo_embedding(ip, bits, ids.numel(), table.data_ptr(), code(table, "table"), table.size(0), width, real(a[2]), y.data, y.stride,
                     code(out, "out"), at.stream),
        "embedding");
  return THPVariable_Wrap(out);
  END_HANDLE_TH_ERRORS
}

// embedding_grad(dout, ids, vocab, scale, dtype, out, accumulate, stream)
PyObject* embedding_grad(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  count(n, 8);
  const at::Tensor& ids = tensor(a[1], "ids");
  const Place at(ids, a[7]);
  const auto [ip, bits] = ids_of(ids);
  const Dense dout(a[0], "dout");
  if (dout->dim() < 1) refuse(PyExc_ValueError, "dout: one dimension at least");
  const int64_t width = dout->sizes().back(), vocab = integer(a[2]), tokens = ids.numel();
  const Rows g = rows_of(*dout, with_width(ids, width), dout->scalar_type(), at.index, "dout");
  const bool accumulate = truth(a[6]);
  at::Tensor out;
  if (a[5] == Py_None) {
    if (accumulate) refuse(PyExc_ValueError, "accumulate: out holds what is added to");
    if (vocab < 0) refuse(PyExc_ValueError, "vocab: negative");
    out = at.empty({vocab, width}, dtype_of(a[4], dout->scalar_type()));
  } else {
    out = tensor(a[5], "out");
    if (out.dim() != 2 || out.size(0) != vocab || out.size(1) != width || !out.is_contiguous() || out.get_device() != at.index)
      refuse(PyExc_ValueError, "out: a contiguous matrix [vocab, width] on the ids' device");
  }
  const int64_t need = fo_embedding_workspace(tokens, width);
  if (need < 0) check(FO_ERR_ARG, "embedding_grad");
  const at::Tensor ws = at.empty({need}, ScalarType::Byte);
  check(fo_embedding_grad(g.data, g.stride, code(*dout, "dout"), ip, bits, tokens, out.data_ptr(), code(out, "out"), vocab, width,
                          real(a[3]), accumulate, ws.data_ptr(), need, at.stream),
        "embedding_grad");
  return THPVariable_Wrap(out);
  END_HANDLE_TH_ERRORS
}

std::pair<void*, int> weight_of(const TensorBase& w, int64_t cols, int device) {
  if (w.dim() != 1 || w.size(0) != cols || w.get_device() != device || !w.is_contiguous())
    refuse(PyExc_ValueError, "weight: a contiguous vector as long as x's last dimension, on x's device");
  return {w.data_ptr(), code(w, "weight")};
}

// The norm, with y and r, or with the 8-bit form, or with both.
PyObject* norm(PyObject* x_, PyObject* residual_, PyObject* weight_, PyObject* eps, PyObject* out_, PyObject* sum_, bool eight, bool with_y,
               PyObject* stream) {
  const at::Tensor &x = tensor(x_, "x"), &weight = tensor(weight_, "weight");
  const int dtype = code(x, "x");
  const Place at(x, stream);
  const at::IntArrayRef shape = x.sizes();
  if (shape.empty()) refuse(PyExc_ValueError, "x: one dimension at least");
  const ScalarType type = x.scalar_type();
  const int64_t cols = shape.back(), rows = cols ? x.numel() / cols : 0;
  const auto [wp, wt] = weight_of(weight, cols, at.index);
  const Rows xr = rows_of(x, shape, type, at.index, "x");
  Rows rr, sr, yr;
  at::Tensor s = x, y, r, q, scales;
  if (residual_ != Py_None) rr = rows_of(tensor(residual_, "residual"), shape, type, at.index, "residual");
  if (residual_ != Py_None || sum_ != Py_None) {
    s = sum_ == Py_None ? at.empty(shape, type) : tensor(sum_, "sum_out");
    sr = rows_of(s, shape, type, at.index, "sum_out");
  }
  const at::IntArrayRef outer = shape.slice(0, shape.size() - 1);
  if (with_y) {
    y = out_ == Py_None ? at.empty(shape, type) : tensor(out_, "out");
    yr = rows_of(y, shape, type, at.index, "out");
    if (!sr.data && yr.data == xr.data && rows > 0) refuse(PyExc_ValueError, "out: x is the sum that is returned; sum_out can take it");
    r = at.empty(outer, ScalarType::Float);
  }
  if (eight) {
    q = at.empty(shape, ScalarType::Float8_e4m3fn);
    at::DimVector groups(outer.begin(), outer.end());
    groups.push_back((cols + 31) / 32);
    scales = at.empty(groups, ScalarType::Byte);
  }
  check(fo_rms_norm(xr.data, xr.stride, rr.data, rr.stride, wp, wt, sr.data, sr.stride, yr.data, yr.stride,
                    eight ? static_cast<uint8_t*>(q.data_ptr()) : nullptr, eight ? static_cast<uint8_t*>(scales.data_ptr()) : nullptr,
                    with_y ? static_cast<float*>(r.data_ptr()) : nullptr, dtype, rows, cols, real(eps), at.stream),
        "rms_norm");
  if (!eight) return tuple({&y, &s, &r});
  return with_y ? tuple({&q, &scales, &y, &s, &r}) : tuple({&q, &scales, &s});
}
// rms_norm(x, residual, weight, eps, out, sum_out, stream)
PyObject* rms_norm(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  count(n, 7);
  return norm(a[0], a[1], a[2], a[3], a[4], a[5], false, true, a[6]);
  END_HANDLE_TH_ERRORS
}
// rms_norm_8bit(x, residual, weight, eps, with_y, stream)
PyObject* rms_norm_8bit(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  count(n, 6);
  return norm(a[0], a[1], a[2], a[3], Py_None, Py_None, true, truth(a[4]), a[5]);
  END_HANDLE_TH_ERRORS
}

// rms_norm_grad(dy, ds, s, weight, r, out, stream)
PyObject* rms_norm_grad(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  count(n, 7);
  const at::Tensor &s = tensor(a[2], "s"), &weight = tensor(a[3], "weight"), &r = tensor(a[4], "r");
  const int dtype = code(s, "s");
  const Place at(s, a[6]);
  const at::IntArrayRef shape = s.sizes();
  if (shape.empty()) refuse(PyExc_ValueError, "s: one dimension at least");
  const ScalarType type = s.scalar_type();
  const int64_t cols = shape.back(), rows = cols ? s.numel() / cols : 0;
  const auto [wp, wt] = weight_of(weight, cols, at.index);
  const Dense dy(a[0], "dy");
  const Rows gr = rows_of(*dy, shape, type, at.index, "dy"), sr = rows_of(s, shape, type, at.index, "s");
  std::optional<Dense> ds;
  Rows dr;
  if (a[1] != Py_None) {
    ds.emplace(a[1], "ds");
    dr = rows_of(**ds, shape, type, at.index, "ds");
  }
  const float* rp = static_cast<const float*>(small(r, shape.slice(0, shape.size() - 1), ScalarType::Float, at.index, "r"));
  const at::Tensor out = a[5] == Py_None ? at.empty(shape, type) : tensor(a[5], "out");
  const Rows xr = rows_of(out, shape, type, at.index, "out");
  const at::Tensor dw = at.empty(weight.sizes(), weight.scalar_type());
  const int64_t need = fo_rms_norm_workspace(rows, cols);
  if (need < 0) check(FO_ERR_ARG, "rms_norm_grad");
  const at::Tensor ws = at.empty({need}, ScalarType::Byte);
  check(fo_rms_norm_grad(gr.data, gr.stride, dr.data, dr.stride, sr.data, sr.stride, wp, wt, rp, xr.data, xr.stride, dw.data_ptr(), dtype,
                         rows, cols, ws.data_ptr(), need, at.stream),
        "rms_norm_grad");
  return tuple({&out, &dw});
  END_HANDLE_TH_ERRORS
}

// decode_8bit(q, scales, dtype, out, stream)
PyObject* decode_8bit(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  count(n, 5);
  const at::Tensor &q = tensor(a[0], "q"), &scales = tensor(a[1], "scales");
  const Place at(q, a[4]);
  const at::IntArrayRef shape = q.sizes();
  if (q.scalar_type() != ScalarType::Float8_e4m3fn || !q.is_contiguous() || shape.empty())
    refuse(PyExc_ValueError, "q: a contiguous float8_e4m3fn tensor of one dimension at least");
  const int64_t cols = shape.back();
  at::DimVector groups(shape.begin(), shape.end() - 1);
  groups.push_back((cols + 31) / 32);
  const void* sp = small(scales, groups, ScalarType::Byte, at.index, "scales");
  const at::Tensor out = a[3] == Py_None ? at.empty(shape, dtype_of(a[2], ScalarType::BFloat16)) : tensor(a[3], "out");
  const Rows y = rows_of(out, shape, out.scalar_type(), at.index, "out");
  check(fo_decode_8bit(static_cast<const uint8_t*>(q.data_ptr()), static_cast<const uint8_t*>(sp), y.data, y.stride, code(out, "out"),
                       cols ? q.numel() / cols : 0, cols, at.stream),
        "decode_8bit");
  return THPVariable_Wrap(out);
  END_HANDLE_TH_ERRORS
}

// A list or tuple of as many items as `want`.
struct Items {
  THPObjectPtr fast;
  Py_ssize_t n;
  Items(PyObject* o, Py_ssize_t want, const char* name) : fast(PySequence_Fast(o, name)) {
    if (!fast) throw python_error();
    n = PySequence_Fast_GET_SIZE(fast.get());
    if (want >= 0 && n != want) refuse(PyExc_ValueError, "%s: as many as updates", name);
  }
  PyObject* operator[](Py_ssize_t i) const { return PySequence_Fast_GET_ITEM(fast.get(), i); }
};

// orthogonalize(grads, momenta, outs, params, step_sizes, steps, coefficients, eps, mu, nesterov, decay, stream); momenta, outs and params
// may be None, outs True to make them.  Returns the list of outs, or None.
PyObject* orthogonalize(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  count(n, 12);
  const Items grads(a[0], -1, "updates: a list of matrices");
  const Py_ssize_t m = grads.n;
  if (m == 0) refuse(PyExc_ValueError, "updates: none");
  const bool make = a[2] == Py_True;
  std::optional<Items> momenta, outs, params, sizes;
  if (a[1] != Py_None) momenta.emplace(a[1], m, "momenta");
  if (a[2] != Py_None && !make) outs.emplace(a[2], m, "out");
  if (a[3] != Py_None) {
    params.emplace(a[3], m, "params");
    sizes.emplace(a[4], m, "scales");
  }
  const Items three(a[6], 3, "coefficients");
  double c[3];
  for (int i = 0; i < 3; ++i) c[i] = real(three[i]);
  const at::Tensor& first = tensor(grads[0], "updates");
  const int dtype = code(first, "updates");
  const ScalarType type = first.scalar_type();
  const Place at(first, a[11]);
  std::vector<fo_matrix_update> items(size_t(m), fo_matrix_update{});
  std::vector<Dense> dense;
  std::vector<at::Tensor> made;
  dense.reserve(size_t(m));
  made.reserve(size_t(m));
  for (Py_ssize_t i = 0; i < m; ++i) {
    dense.emplace_back(grads[i], "updates");
    const at::Tensor& g = *dense.back();
    if (g.dim() != 2) refuse(PyExc_ValueError, "updates: matrices");
    const at::IntArrayRef shape = g.sizes();
    fo_matrix_update& it = items[size_t(i)];
    it.rows = shape[0];
    it.cols = shape[1];
    const Rows gr = rows_of(g, shape, type, at.index, "updates");
    it.grad = gr.data;
    it.grad_stride = gr.stride;
    if (momenta) {
      const Rows r = rows_of(tensor((*momenta)[i], "momenta"), shape, ScalarType::Float, at.index, "momenta");
      it.momentum = static_cast<float*>(r.data);
      it.momentum_stride = r.stride;
    }
    if (make || outs) {
      if (make) made.push_back(at.empty(shape, type));
      const Rows r = rows_of(make ? made.back() : tensor((*outs)[i], "out"), shape, type, at.index, "out");
      it.out = r.data;
      it.out_stride = r.stride;
    }
    if (params) {
      const Rows r = rows_of(tensor((*params)[i], "params"), shape, ScalarType::Float, at.index, "params");
      it.param = static_cast<float*>(r.data);
      it.param_stride = r.stride;
      it.step = float(real((*sizes)[i]));
    }
  }
  const int64_t need = fo_orthogonalize_workspace(items.data(), int(m), dtype);
  if (need < 0) check(FO_ERR_ARG, "orthogonalize");
  const at::Tensor ws = at.empty({need}, ScalarType::Byte);
  const int64_t steps = integer(a[5]);
  check(fo_orthogonalize(items.data(), int(m), dtype, int(steps < 0 ? 0 : steps > 65 ? 65 : steps), c, real(a[7]), real(a[8]), truth(a[9]),
                         real(a[10]), ws.data_ptr(), need, at.stream),
        "orthogonalize");
  if (!make) Py_RETURN_NONE;
  THPObjectPtr list(PyList_New(m));
  if (!list) throw python_error();
  for (Py_ssize_t i = 0; i < m; ++i) {
    PyObject* o = THPVariable_Wrap(made[size_t(i)]);
    if (!o) throw python_error();
    PyList_SET_ITEM(list.get(), i, o);
  }
  return list.release();
  END_HANDLE_TH_ERRORS
}

PyObject* set_error(PyObject*, PyObject* cls) {
  Py_INCREF(cls);
  Py_XDECREF(g_error);
  g_error = cls;
  Py_RETURN_NONE;
}

template <typename F>
PyCFunction fast(F f) {
  return reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(f));
}
PyMethodDef methods[] = {{"embedding", fast(embedding), METH_FASTCALL, nullptr},
                         {"embedding_grad", fast(embedding_grad), METH_FASTCALL, nullptr},
                         {"rms_norm", fast(rms_norm), METH_FASTCALL, nullptr},
                         {"rms_norm_8bit", fast(rms_norm_8bit), METH_FASTCALL, nullptr},
                         {"rms_norm_grad", fast(rms_norm_grad), METH_FASTCALL, nullptr},
                         {"decode_8bit", fast(decode_8bit), METH_FASTCALL, nullptr},
                         {"orthogonalize", fast(orthogonalize), METH_FASTCALL, nullptr},
                         {"set_error", set_error, METH_O, nullptr},
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_binding", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__binding() { return PyModule_Create(&module); }

// The layer operators on torch tensors: argument checks, allocation of outputs and workspaces, the call into libsds.
// Small calls run for two or three microseconds on the GPU; the same checks through the interpreter and ctypes took
// eight to thirty. Positional arguments only; layers.py holds the signatures and their documentation.
#include <Python.h>

#include <ATen/cuda/EmptyTensor.h>
#include <c10/core/GradMode.h>
#include <c10/cuda/CUDAGuard.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/Dtype.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include <stdexcept>
#include <string>

#include "../../include/sds.h"

namespace {

// a bad argument: ValueError; a code from the library: SdsError (set as Python error by the thrower)
struct BadArgument : std::runtime_error {
  using std::runtime_error::runtime_error;
};
struct PythonError {};

void require(bool ok, const char* what) {
  if (!ok) throw BadArgument(what);
}

void check(int rc, const char* where) {
  if (rc == SDS_OK) return;
  PyObject* mod = PyImport_ImportModule("paper_2501_05370_b200.binding");
  PyObject* cls = mod ? PyObject_GetAttrString(mod, "SdsError") : nullptr;
  PyObject* err = cls ? PyObject_CallFunction(cls, "is", rc, where) : nullptr;
  if (err) PyErr_SetObject(cls, err);
  Py_XDECREF(err);
  Py_XDECREF(cls);
  Py_XDECREF(mod);
  throw PythonError{};
}

const at::Tensor& tensor(PyObject* o, const char* what) {
  if (!THPVariable_Check(o)) throw BadArgument(std::string(what) + " must be a torch tensor");
  return THPVariable_Unpack(o);
}

int type_code(at::ScalarType t) {
  switch (t) {
    case at::kFloat: return SDS_F32;
    case at::kBFloat16: return SDS_BF16;
    case at::kHalf: return SDS_F16;
    default: throw BadArgument(std::string("unsupported dtype ") + c10::toString(t));
  }
}

// a CUDA tensor [..., d] whose leading dimensions make evenly spaced rows
struct Rows {
  int64_t rows, d, ld;
};
Rows rows_of(const at::Tensor& x, const char* what) {
  const std::string name(what);
  if (!x.is_cuda()) throw BadArgument(name + " must be a CUDA tensor");
  const auto sizes = x.sizes();
  const auto strides = x.strides();
  const int64_t n = x.dim();
  if (n < 1 || sizes[n - 1] < 1 || sizes[n - 1] > INT32_MAX) throw BadArgument(name + " must be [..., d]");
  Rows r{x.numel() / sizes[n - 1], sizes[n - 1], sizes[n - 1]};
  if (x.is_contiguous() || r.rows == 0) return r;
  if (r.d > 1 && strides[n - 1] != 1) throw BadArgument(name + " must be contiguous along its last dimension");
  int64_t ld = -1, span = 1;                       // span: rows covered by the dimensions seen so far, innermost first
  for (int64_t k = n - 2; k >= 0; --k) {
    if (sizes[k] == 1) continue;
    if (ld < 0) ld = strides[k];
    else if (strides[k] != ld * span) throw BadArgument(name + ": the leading dimensions must be evenly spaced rows");
    span *= sizes[k];
  }
  if (ld >= 0) r.ld = ld;
  if (r.ld < r.d) throw BadArgument(name + ": rows must not overlap (call contiguous() on broadcast rows)");
  return r;
}

const void* vector_of(PyObject* o, int64_t d, const at::Tensor& x, const char* what, at::ScalarType* type) {
  if (o == Py_None) return nullptr;
  const at::Tensor& v = tensor(o, what);
  if (v.dim() != 1 || v.numel() != d || !v.is_contiguous() || v.device() != x.device())
    throw BadArgument(std::string(what) + " must be a contiguous vector of x's last size on x's device");
  *type = v.scalar_type();
  return v.data_ptr();
}

at::Tensor empty(at::IntArrayRef sizes, at::ScalarType type, const at::Tensor& like) {
  return at::detail::empty_cuda(sizes, type, like.device(), std::nullopt);
}

// the caller's tensor for the output, or a new one
at::Tensor output(PyObject* o, const at::Tensor& x, at::ScalarType type, int64_t* ld) {
  if (o == Py_None) {
    *ld = x.size(-1);
    return empty(x.sizes(), type, x);
  }
  const at::Tensor& y = tensor(o, "out");
  require(y.sizes() == x.sizes() && y.scalar_type() == type && y.device() == x.device(),
          "out must have x's shape and device and the output's type");
  *ld = rows_of(y, "out").ld;
  return y;
}

at::ScalarType dtype_or(PyObject* o, at::ScalarType other) {
  if (o == Py_None) return other;
  require(THPDtype_Check(o), "out_dtype must be a torch dtype");
  return reinterpret_cast<THPDtype*>(o)->scalar_type;
}

// x's leading dimensions with n columns
bool has_shape(const at::Tensor& y, const at::Tensor& x, int64_t n) {
  return y.dim() == x.dim() && y.size(-1) == n && y.sizes().slice(0, y.dim() - 1) == x.sizes().slice(0, x.dim() - 1);
}

// what Python says of a number that is none, or too large, is a bad argument here
[[noreturn]] void bad_number(const char* what) {
  if (!PyErr_ExceptionMatches(PyExc_TypeError) && !PyErr_ExceptionMatches(PyExc_OverflowError) && !PyErr_ExceptionMatches(PyExc_ValueError))
    throw PythonError{};
  PyErr_Clear();
  throw BadArgument(what);
}
int64_t integer(PyObject* o, const char* what) {
  const long long v = PyLong_AsLongLong(o);
  if (v == -1 && PyErr_Occurred()) bad_number(what);
  return v;
}

at::Tensor workspace(PyObject* o, size_t need, const at::Tensor& x) {
  if (o == Py_None) return empty({(int64_t)need}, at::kByte, x);
  const at::Tensor& w = tensor(o, "workspace");
  if (w.scalar_type() != at::kByte || w.device() != x.device() || !w.is_contiguous() || (size_t)w.numel() < need)
    throw BadArgument("workspace must be a contiguous uint8 tensor of at least " + std::to_string(need) + " bytes on x's device");
  return w;
}

bool truth(PyObject* o) {
  const int r = PyObject_IsTrue(o);
  if (r < 0) throw PythonError{};
  return r != 0;
}

// the k-th truth value of `want`
bool wanted(PyObject* want, Py_ssize_t k, Py_ssize_t n) {
  PyObject* fast = PySequence_Fast(want, "want must be a sequence of truth values");
  if (!fast) throw PythonError{};
  const bool right = PySequence_Fast_GET_SIZE(fast) == n;
  const int r = right ? PyObject_IsTrue(PySequence_Fast_GET_ITEM(fast, k)) : 0;
  Py_DECREF(fast);
  if (r < 0) throw PythonError{};
  require(right, "want must hold one truth value per gradient");
  return r != 0;
}

// Nothing is recorded for autograd: a warning, at the line that called layers.py, where torch would have recorded something.
void warn_unrecorded(const char* name, std::initializer_list<PyObject*> inputs) {
  const bool recording = c10::GradMode::is_enabled();
  for (PyObject* o : inputs) {
    if (o == Py_None) continue;
    const at::Tensor& t = THPVariable_Unpack(o);
    if (!(recording && t.requires_grad()) && !t._fw_grad(0).defined()) continue;
    const std::string what = std::string(name) + " records nothing for autograd, and an input requires a gradient: call " + name +
                             "_backward for it, and " + name + " under torch.no_grad() or on detached tensors";
    if (PyErr_WarnEx(PyExc_UserWarning, what.c_str(), 2) != 0) throw PythonError{};
    return;
  }
}

PyObject* wrap(const at::Tensor& t) {
  if (!t.defined()) Py_RETURN_NONE;
  return THPVariable_Wrap(t);
}
PyObject* tuple(std::initializer_list<at::Tensor> ts) {
  PyObject* r = PyTuple_New((Py_ssize_t)ts.size());
  if (!r) throw PythonError{};
  Py_ssize_t i = 0;
  for (const at::Tensor& t : ts) {
    PyObject* o = wrap(t);
    if (!o) {
      Py_DECREF(r);
      throw PythonError{};
    }
    PyTuple_SET_ITEM(r, i++, o);
  }
  return r;
}

void* ptr(const at::Tensor& t) { return t.defined() ? t.data_ptr() : nullptr; }

template <class F>
PyObject* guarded(Py_ssize_t n, Py_ssize_t want, F f) {
  if (n != want) {
    PyErr_SetString(PyExc_TypeError, "wrong number of arguments");
    return nullptr;
  }
  try {
    return f();
  } catch (const PythonError&) {
  } catch (const BadArgument& e) {
    PyErr_SetString(PyExc_ValueError, e.what());
  } catch (...) {                                  // torch's own, an allocation that failed among them
    torch::translate_exception_to_python(std::current_exception());
  }
  return nullptr;
}

// ---------------------------------------------------------------------------------------------
// layer norm
// ---------------------------------------------------------------------------------------------

// (x, weight, bias, eps, out_dtype, stats, out)
PyObject* layer_norm(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded(n, 7, [&]() -> PyObject* {
    const at::Tensor& x = tensor(a[0], "x");
    const Rows r = rows_of(x, "x");
    at::ScalarType wt = at::kFloat, bt = at::kFloat, yt = x.scalar_type();
    const void* w = vector_of(a[1], r.d, x, "weight", &wt);
    const void* b = vector_of(a[2], r.d, x, "bias", &bt);
    require(!w || !b || wt == bt, "weight and bias must have the same type");
    const double eps = PyFloat_AsDouble(a[3]);
    if (eps == -1.0 && PyErr_Occurred()) throw PythonError{};
    if (a[4] != Py_None) {
      require(THPDtype_Check(a[4]), "out_dtype must be a torch dtype");
      yt = reinterpret_cast<THPDtype*>(a[4])->scalar_type;
    }
    const int tx = type_code(x.scalar_type()), ty = type_code(yt), tw = type_code(w ? wt : bt);
    warn_unrecorded("layer_norm", {a[0], a[1], a[2]});
    const c10::cuda::CUDAGuard guard(x.device());
    int64_t ldy = 0;
    const at::Tensor y = output(a[6], x, yt, &ldy);
    at::Tensor mean, rstd;
    if (truth(a[5])) {
      const auto lead = x.sizes().slice(0, x.dim() - 1);
      mean = empty(lead, at::kFloat, x);
      rstd = empty(lead, at::kFloat, x);
    }
    check(sds_layer_norm(x.data_ptr(), r.ld, tx, w, b, tw, r.rows, (int32_t)r.d, (float)eps, y.data_ptr(), ldy, ty,
                         static_cast<float*>(ptr(mean)), static_cast<float*>(ptr(rstd)),
                         c10::cuda::getCurrentCUDAStream(x.get_device()).stream()),
          "sds_layer_norm");
    return mean.defined() ? tuple({y, mean, rstd}) : wrap(y);
  });
}

// (dy, x, weight, mean, rstd, want, workspace)
PyObject* layer_norm_backward(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded(n, 7, [&]() -> PyObject* {
    const at::Tensor &dy = tensor(a[0], "dy"), &x = tensor(a[1], "x"), &mean = tensor(a[3], "mean"), &rstd = tensor(a[4], "rstd");
    const Rows r = rows_of(x, "x");
    require(dy.sizes() == x.sizes() && dy.device() == x.device(), "dy must have x's shape and device");
    const int64_t lddy = rows_of(dy, "dy").ld;
    at::ScalarType wt = at::kFloat;
    const void* w = vector_of(a[2], r.d, x, "weight", &wt);
    for (const at::Tensor* v : {&mean, &rstd})
      require(v->scalar_type() == at::kFloat && v->numel() == r.rows && v->is_contiguous() && v->device() == x.device(),
              "mean and rstd must be contiguous float32 tensors with one value per row, on x's device");
    const int tx = type_code(x.scalar_type()), ty = type_code(dy.scalar_type()), tw = type_code(wt);
    const c10::cuda::CUDAGuard guard(x.device());
    at::Tensor dx, dw, db;
    if (wanted(a[5], 0, 3)) dx = empty(x.sizes(), x.scalar_type(), x);
    if (wanted(a[5], 1, 3)) dw = empty({r.d}, wt, x);
    if (wanted(a[5], 2, 3)) db = empty({r.d}, wt, x);
    size_t need = 0;
    check(sds_layer_norm_workspace_bytes(r.rows, (int32_t)r.d, &need), "sds_layer_norm_workspace_bytes");
    const at::Tensor ws = workspace(a[6], need, x);
    check(sds_layer_norm_backward(dy.data_ptr(), lddy, ty, x.data_ptr(), r.ld, tx, w, tw, mean.data_ptr<float>(),
                                  rstd.data_ptr<float>(), r.rows, (int32_t)r.d, ptr(dx), r.d, ptr(dw), ptr(db),
                                  ws.data_ptr(), (size_t)ws.numel(),
                                  c10::cuda::getCurrentCUDAStream(x.get_device()).stream()),
          "sds_layer_norm_backward");
    return tuple({dx, dw, db});
  });
}

// ---------------------------------------------------------------------------------------------
// gated feed-forward block
// ---------------------------------------------------------------------------------------------

struct Ffn {
  Rows r;
  int64_t f;
  int type;
  sds_gated_ffn_sizes sizes;
};
Ffn ffn_of(const at::Tensor& x, const at::Tensor& wg, const at::Tensor& wu, const at::Tensor& wd) {
  Ffn s{};
  s.r = rows_of(x, "x");
  s.f = wg.dim() == 2 ? wg.size(0) : -1;
  const int64_t d = s.r.d, f = s.f;
  require(f > 0 && f <= INT32_MAX && wg.sizes() == at::IntArrayRef({f, d}) && wu.sizes() == at::IntArrayRef({f, d}) &&
              wd.sizes() == at::IntArrayRef({d, f}),
          "w_gate and w_up must be [f, d] and w_down [d, f] for x [..., d]");
  for (const at::Tensor* w : {&wg, &wu, &wd})
    require(w->scalar_type() == x.scalar_type() && w->device() == x.device() && w->is_contiguous(),
            "the weights must be contiguous tensors of x's type on x's device");
  s.type = type_code(x.scalar_type());
  check(sds_gated_ffn_bytes(s.r.rows, (int32_t)d, (int32_t)f, &s.sizes), "sds_gated_ffn_bytes");
  return s;
}

// (x, w_gate, w_up, w_down, act, keep, out, workspace)
PyObject* gated_ffn(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded(n, 8, [&]() -> PyObject* {
    const at::Tensor &x = tensor(a[0], "x"), &wg = tensor(a[1], "w_gate"), &wu = tensor(a[2], "w_up"), &wd = tensor(a[3], "w_down");
    const Ffn s = ffn_of(x, wg, wu, wd);
    const long act = PyLong_AsLong(a[4]);
    if (act == -1 && PyErr_Occurred()) throw PythonError{};
    const bool keep = truth(a[5]);
    warn_unrecorded("gated_ffn", {a[0], a[1], a[2], a[3]});
    const c10::cuda::CUDAGuard guard(x.device());
    int64_t ldy = 0;
    const at::Tensor y = output(a[6], x, x.scalar_type(), &ldy);
    at::Tensor kept;
    if (keep) kept = empty({(int64_t)s.sizes.keep_bytes}, at::kByte, x);
    const at::Tensor ws = workspace(a[7], keep ? s.sizes.forward_keep_bytes : s.sizes.forward_bytes, x);
    check(sds_gated_ffn(x.data_ptr(), s.r.ld, s.type, s.r.rows, (int32_t)s.r.d, (int32_t)s.f, wg.data_ptr(), wu.data_ptr(),
                        wd.data_ptr(), (int32_t)act, y.data_ptr(), ldy, ptr(kept), ws.data_ptr(), (size_t)ws.numel(),
                        c10::cuda::getCurrentCUDAStream(x.get_device()).stream()),
          "sds_gated_ffn");
    return keep ? tuple({y, kept}) : wrap(y);
  });
}

// (dy, x, w_gate, w_up, w_down, kept, want, workspace)
PyObject* gated_ffn_backward(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded(n, 8, [&]() -> PyObject* {
    const at::Tensor &dy = tensor(a[0], "dy"), &x = tensor(a[1], "x"), &wg = tensor(a[2], "w_gate"), &wu = tensor(a[3], "w_up"),
                     &wd = tensor(a[4], "w_down"), &kept = tensor(a[5], "kept");
    const Ffn s = ffn_of(x, wg, wu, wd);
    require(dy.sizes() == x.sizes() && dy.scalar_type() == x.scalar_type() && dy.device() == x.device(),
            "dy must have x's shape, type and device");
    const int64_t lddy = rows_of(dy, "dy").ld;
    require(kept.scalar_type() == at::kByte && kept.is_contiguous() && kept.device() == x.device() &&
                (size_t)kept.numel() >= s.sizes.keep_bytes,
            "kept must be what gated_ffn(keep=True) returned for these sizes");
    const c10::cuda::CUDAGuard guard(x.device());
    at::Tensor g[4];
    const at::Tensor* like[4] = {&x, &wg, &wu, &wd};
    for (int k = 0; k < 4; ++k)
      if (wanted(a[6], k, 4)) g[k] = empty(like[k]->sizes(), x.scalar_type(), x);
    const at::Tensor ws = workspace(a[7], s.sizes.backward_bytes, x);
    check(sds_gated_ffn_backward(dy.data_ptr(), lddy, x.data_ptr(), s.r.ld, s.type, s.r.rows, (int32_t)s.r.d, (int32_t)s.f,
                                 wg.data_ptr(), wu.data_ptr(), wd.data_ptr(), kept.data_ptr(), ptr(g[0]), s.r.d, ptr(g[1]),
                                 ptr(g[2]), ptr(g[3]), ws.data_ptr(), (size_t)ws.numel(),
                                 c10::cuda::getCurrentCUDAStream(x.get_device()).stream()),
          "sds_gated_ffn_backward");
    return tuple({g[0], g[1], g[2], g[3]});
  });
}

// ---------------------------------------------------------------------------------------------
// linear layer
// ---------------------------------------------------------------------------------------------

struct Linear {
  Rows r;
  sds_linear_layer layer;
  const int32_t* step;
  at::ScalarType bias_type;
};
// the layer of x, weight, bias, table and step (the last three may be None)
Linear linear_of(const at::Tensor& x, const at::Tensor& w, PyObject* bias, PyObject* table, PyObject* step, int act) {
  Linear s{};
  s.r = rows_of(x, "x");
  const at::ScalarType t = x.scalar_type();
  require(w.dim() == 2 && w.size(0) > 0 && w.size(0) <= INT32_MAX && w.size(1) == s.r.d && w.scalar_type() == t && w.device() == x.device() &&
              w.is_contiguous(),
          "weight must be a contiguous [n, k] tensor of x's type on x's device, for x [..., k]");
  const int64_t n = w.size(0);
  s.layer.k = (int32_t)s.r.d; s.layer.n = (int32_t)n;
  s.layer.dtype = type_code(t); s.layer.act = act;
  s.layer.w_dev = w.data_ptr();
  s.bias_type = at::kFloat;
  if (bias != Py_None) {
    const at::Tensor& b = tensor(bias, "bias");
    require(b.dim() == 1 && b.numel() == n && b.is_contiguous() && b.device() == x.device(),
            "bias must be a contiguous vector of the weight's first size on x's device");
    s.bias_type = b.scalar_type();
    s.layer.bias_dev = b.data_ptr();
  }
  s.layer.bias_dtype = type_code(s.bias_type);
  require((table == Py_None) == (step == Py_None), "table and step come together");
  if (table != Py_None) {
    const at::Tensor &v = tensor(table, "table"), &at = tensor(step, "step");
    require(v.dim() == 2 && v.size(0) > 0 && v.size(0) <= INT32_MAX && v.size(1) == n && v.scalar_type() == t && v.device() == x.device() &&
                v.is_contiguous(),
            "table must be a contiguous [steps, n] tensor of x's type on x's device");
    require(at.scalar_type() == at::kInt && at.numel() == s.r.rows && at.is_contiguous() && at.device() == x.device(),
            "step must be a contiguous int32 tensor with one value per row of x, on x's device");
    s.layer.table_dev = v.data_ptr();
    s.layer.steps = (int32_t)v.size(0);
    s.step = at.data_ptr<int32_t>();
  }
  return s;
}

sds_linear_sizes linear_sizes(const Linear& s) {
  sds_linear_sizes sizes;
  check(sds_linear_bytes(&s.layer, s.r.rows, &sizes), "sds_linear_bytes");
  return sizes;
}

// what the forward call returns for the backward one: a single byte that says so where there is nothing to keep
int64_t kept_size(const sds_linear_sizes& sizes) { return sizes.keep_bytes ? (int64_t)sizes.keep_bytes : 1; }

// (x, weight, bias, act, table, step, residual, out_dtype, keep, out, workspace)
PyObject* linear(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded(n, 11, [&]() -> PyObject* {
    const at::Tensor &x = tensor(a[0], "x"), &w = tensor(a[1], "weight");
    const Linear s = linear_of(x, w, a[2], a[4], a[5], (int)integer(a[3], "activation must be a number"));
    const at::ScalarType yt = dtype_or(a[7], x.scalar_type());
    const int ty = type_code(yt);
    const void* residual = nullptr;
    int64_t ldr = 0;
    if (a[6] != Py_None) {
      const at::Tensor& v = tensor(a[6], "residual");
      require(has_shape(v, x, s.layer.n) && v.scalar_type() == yt && v.device() == x.device(),
              "residual must have the output's shape and type and x's device");
      ldr = rows_of(v, "residual").ld;
      residual = v.data_ptr();
    }
    const bool keep = truth(a[8]);
    warn_unrecorded("linear", {a[0], a[1], a[2], a[4], a[6]});
    const sds_linear_sizes sizes = linear_sizes(s);
    const c10::cuda::CUDAGuard guard(x.device());
    at::Tensor y, kept;
    int64_t ldy = s.layer.n;
    if (a[9] == Py_None) {
      c10::SmallVector<int64_t, 8> shape(x.sizes().begin(), x.sizes().end());
      shape.back() = s.layer.n;
      y = empty(shape, yt, x);
    } else {
      y = tensor(a[9], "out");
      require(has_shape(y, x, s.layer.n) && y.scalar_type() == yt && y.device() == x.device(),
              "out must have the output's shape and type and x's device");
      ldy = rows_of(y, "out").ld;
    }
    if (keep) kept = empty({kept_size(sizes)}, at::kByte, x);
    const at::Tensor ws = workspace(a[10], sizes.forward_bytes, x);
    check(sds_linear(&s.layer, x.data_ptr(), s.r.ld, s.step, s.r.rows, residual, ldr, y.data_ptr(), ldy, ty,
                     sizes.keep_bytes ? ptr(kept) : nullptr, ws.data_ptr(), (size_t)ws.numel(),
                     c10::cuda::getCurrentCUDAStream(x.get_device()).stream()),
          "sds_linear");
    return keep ? tuple({y, kept}) : wrap(y);
  });
}

// (dy, x, weight, kept, bias, table, step, want, workspace)
PyObject* linear_backward(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded(n, 9, [&]() -> PyObject* {
    const at::Tensor &dy = tensor(a[0], "dy"), &x = tensor(a[1], "x"), &w = tensor(a[2], "weight"), &kept = tensor(a[3], "kept");
    // (which activation it was is in what the forward call kept: one byte, without one)
    const Linear s = linear_of(x, w, a[4], a[5], a[6], kept.numel() != 1 ? SDS_ACT_SILU : SDS_ACT_NONE);
    require(has_shape(dy, x, s.layer.n) && dy.device() == x.device(), "dy must have the output's shape and x's device");
    const int64_t lddy = rows_of(dy, "dy").ld;
    const int ty = type_code(dy.scalar_type());
    const sds_linear_sizes sizes = linear_sizes(s);
    require(kept.scalar_type() == at::kByte && kept.is_contiguous() && kept.device() == x.device() &&
                kept.numel() == kept_size(sizes),
            "kept must be what linear(keep=True) returned for these sizes");
    const c10::cuda::CUDAGuard guard(x.device());
    at::Tensor g[4];
    if (wanted(a[7], 0, 4)) g[0] = empty(x.sizes(), x.scalar_type(), x);
    if (wanted(a[7], 1, 4)) g[1] = empty(w.sizes(), x.scalar_type(), x);
    if (wanted(a[7], 2, 4) && s.layer.bias_dev) g[2] = empty({s.layer.n}, s.bias_type, x);
    if (wanted(a[7], 3, 4) && s.layer.table_dev) g[3] = empty({s.layer.steps, s.layer.n}, x.scalar_type(), x);
    const at::Tensor ws = workspace(a[8], sizes.backward_bytes, x);
    check(sds_linear_backward(&s.layer, dy.data_ptr(), lddy, ty, x.data_ptr(), s.r.ld, s.step, s.r.rows, sizes.keep_bytes ? kept.data_ptr() : nullptr,
                              ptr(g[0]), s.r.d, ptr(g[1]), ptr(g[2]), ptr(g[3]), ws.data_ptr(), (size_t)ws.numel(),
                              c10::cuda::getCurrentCUDAStream(x.get_device()).stream()),
          "sds_linear_backward");
    return tuple({g[0], g[1], g[2], g[3]});
  });
}

// ---------------------------------------------------------------------------------------------
// dropout
// ---------------------------------------------------------------------------------------------

double real(PyObject* o, const char* what) {
  const double v = PyFloat_AsDouble(o);
  if (v == -1.0 && PyErr_Occurred()) bad_number(what);
  return v;
}

// a[0..3] = p, seed, step (a number, or an int32 tensor of one element on x's device), row0
sds_dropout_spec dropout_of(PyObject* const* a, const at::Tensor& x) {
  sds_dropout_spec s{};
  s.p = real(a[0], "p must be a number");
  PyObject* seed = PyNumber_Index(a[1]);
  s.seed = seed ? PyLong_AsUnsignedLongLong(seed) : (uint64_t)-1;
  Py_XDECREF(seed);
  if (s.seed == (uint64_t)-1 && PyErr_Occurred()) bad_number("seed must be an integer in [0, 2^64)");
  if (THPVariable_Check(a[2])) {
    const at::Tensor& t = THPVariable_Unpack(a[2]);
    require(t.scalar_type() == at::kInt && t.numel() == 1 && t.device() == x.device(),
            "step must be a number or an int32 tensor of one element on x's device");
    s.step_dev = t.data_ptr<int32_t>();
  } else {
    const int64_t step = integer(a[2], "step must be in [0, 2^31), or an int32 tensor of one element on x's device");
    require(step >= 0 && step <= INT32_MAX, "step must be in [0, 2^31)");
    s.step = (int32_t)step;
  }
  s.row0 = integer(a[3], "row0 must be an integer below 2^56");
  require(s.p >= 0.0 && s.p <= 1.0, "p must be in [0, 1]");
  require(s.row0 >= 0, "row0 must not be negative");
  return s;
}

// (x, p, seed, step, row0, residual, out_dtype, out)
PyObject* dropout(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded(n, 8, [&]() -> PyObject* {
    const at::Tensor& x = tensor(a[0], "x");
    const Rows r = rows_of(x, "x");
    const sds_dropout_spec spec = dropout_of(a + 1, x);
    const int tx = type_code(x.scalar_type());
    at::ScalarType yt = dtype_or(a[6], x.scalar_type());
    const void* residual = nullptr;
    int64_t ldr = 0;
    if (a[5] != Py_None) {
      const at::Tensor& v = tensor(a[5], "residual");
      require(v.sizes() == x.sizes() && v.device() == x.device(), "residual must have x's shape and device");
      yt = v.scalar_type();
      ldr = rows_of(v, "residual").ld;
      residual = v.data_ptr();
    }
    const int ty = type_code(yt);
    warn_unrecorded("dropout", {a[0], a[5]});
    const c10::cuda::CUDAGuard guard(x.device());
    int64_t ldy = 0;
    const at::Tensor y = output(a[7], x, yt, &ldy);
    check(sds_dropout(&spec, x.data_ptr(), r.ld, tx, r.rows, (int32_t)r.d, residual, ldr, y.data_ptr(), ldy, ty,
                      c10::cuda::getCurrentCUDAStream(x.get_device()).stream()),
          "sds_dropout");
    return wrap(y);
  });
}

// ---------------------------------------------------------------------------------------------
// residual norm
// ---------------------------------------------------------------------------------------------

struct ResidualNorm {
  sds_residual_norm_op op;
  Rows r;
  at::ScalarType w_type, c_type;
  const at::Tensor* cond[3];                       // gate, scale, shift
  const at::Tensor* h;
  int64_t ldh;
};
// a[0..13] = weight, bias, scale, shift, gate, post, post_weight, rms, alpha, eps, p, seed, step, row0
ResidualNorm residual_norm_of(const at::Tensor& r, PyObject* h, at::ScalarType n_type, PyObject* const* a) {
  ResidualNorm s{};
  s.r = rows_of(r, "r");
  const int64_t d = s.r.d;
  sds_residual_norm_op& op = s.op;
  op.rows = s.r.rows; op.d = (int32_t)d; op.groups = 1;
  op.r_dtype = type_code(r.scalar_type()); op.h_dtype = type_code(n_type);
  if (h != Py_None) {
    s.h = &tensor(h, "h");
    require(s.h->sizes() == r.sizes() && s.h->device() == r.device() && s.h->scalar_type() == n_type,
            "h must have r's shape and device and the type of n");
    s.ldh = rows_of(*s.h, "h").ld;
  }
  op.post = truth(a[5]);
  const struct { PyObject* o; const char* name; const void** to; } vectors[3] = {
      {a[0], "weight", &op.w_dev}, {a[1], "bias", &op.b_dev}, {a[6], "post_weight", &op.post_w_dev}};
  s.w_type = at::kFloat;
  bool first = true;
  for (const auto& v : vectors) {
    at::ScalarType t = s.w_type;
    *v.to = vector_of(v.o, d, r, v.name, &t);
    if (!*v.to) continue;
    require(first || t == s.w_type, "weight, bias and post_weight must have the same type");
    s.w_type = t;
    first = false;
  }
  require(op.post || !op.post_w_dev, "post_weight needs post=True");
  op.w_dtype = type_code(s.w_type);
  const struct { PyObject* o; const char* name; const void** to; int64_t* ld; } conds[3] = {
      {a[4], "gate", &op.gate_dev, &op.ld_gate}, {a[2], "scale", &op.scale_dev, &op.ld_scale}, {a[3], "shift", &op.shift_dev, &op.ld_shift}};
  s.c_type = at::kFloat;
  first = true;
  for (int k = 0; k < 3; ++k) {
    if (conds[k].o == Py_None) continue;
    const at::Tensor& t = tensor(conds[k].o, conds[k].name);
    const Rows g = rows_of(t, conds[k].name);
    require(t.device() == r.device() && g.d == d && g.rows > 0 && (first || (g.rows == op.groups && t.scalar_type() == s.c_type)),
            "gate, scale and shift must be [groups, d] tensors of one type on r's device, with r's last size");
    op.groups = g.rows;
    *conds[k].to = t.data_ptr();
    *conds[k].ld = g.ld;
    s.c_type = t.scalar_type();
    s.cond[k] = &t;
    first = false;
  }
  require(op.rows % op.groups == 0, "the rows of r must be a multiple of the rows of gate, scale and shift");
  require(s.h || (!s.cond[0] && !op.post), "gate and post need h");
  op.cond_dtype = type_code(s.c_type);
  op.kind = truth(a[7]) ? SDS_NORM_RMS : SDS_NORM_LAYER;
  op.alpha = (float)real(a[8], "alpha must be a number");
  op.eps = (float)real(a[9], "eps must be a number");
  op.drop = dropout_of(a + 10, r);
  require(s.h || op.drop.p == 0.0, "dropout needs h");
  return s;
}

// (r, h, [14 of residual_norm_of], out_dtype, keep, out, stream_out)
PyObject* residual_norm(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded(n, 20, [&]() -> PyObject* {
    const at::Tensor& r = tensor(a[0], "r");
    const at::ScalarType other = a[1] == Py_None ? r.scalar_type() : tensor(a[1], "h").scalar_type();
    const at::ScalarType nt = dtype_or(a[16], other);
    const ResidualNorm s = residual_norm_of(r, a[1], nt, a + 2);
    const bool keep = truth(a[17]);
    warn_unrecorded("residual_norm", {a[0], a[1], a[2], a[3], a[4], a[5], a[6], a[8]});
    sds_residual_norm_sizes sizes;
    check(sds_residual_norm_bytes(&s.op, &sizes), "sds_residual_norm_bytes");
    const c10::cuda::CUDAGuard guard(r.device());
    int64_t ldn = 0, ldo = 0;
    const at::Tensor y = output(a[18], r, nt, &ldn);
    at::Tensor out, kept;
    if (s.h) out = output(a[19], r, r.scalar_type(), &ldo);
    else require(a[19] == Py_None, "stream_out needs h");
    if (keep) kept = empty({s.r.rows, 8}, at::kFloat, r);
    check(sds_residual_norm(&s.op, r.data_ptr(), s.r.ld, s.h ? s.h->data_ptr() : nullptr, s.ldh, ptr(out), ldo, y.data_ptr(), ldn,
                            static_cast<float*>(ptr(kept)), c10::cuda::getCurrentCUDAStream(r.get_device()).stream()),
          "sds_residual_norm");
    const at::Tensor& stream = s.h ? out : r;
    return keep ? tuple({stream, y, kept}) : tuple({stream, y});
  });
}

// (dn, dr, r, h, kept, [14 of residual_norm_of], want, workspace)
PyObject* residual_norm_backward(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded(n, 21, [&]() -> PyObject* {
    const at::Tensor &dn = tensor(a[0], "dn"), &r = tensor(a[2], "r"), &kept = tensor(a[4], "kept");
    const ResidualNorm s = residual_norm_of(r, a[3], dn.scalar_type(), a + 5);
    require(dn.sizes() == r.sizes() && dn.device() == r.device(), "dn must have r's shape and device");
    const int64_t lddn = rows_of(dn, "dn").ld;
    const void* dout = nullptr;
    int64_t lddout = 0;
    if (a[1] != Py_None) {
      const at::Tensor& v = tensor(a[1], "dr");
      require(v.sizes() == r.sizes() && v.device() == r.device() && v.scalar_type() == r.scalar_type(), "dr must have r's shape, type and device");
      lddout = rows_of(v, "dr").ld;
      dout = v.data_ptr();
    }
    require(kept.scalar_type() == at::kFloat && kept.is_contiguous() && kept.device() == r.device() && kept.numel() == 8 * s.r.rows,
            "kept must be what residual_norm(keep=True) returned for these sizes");
    sds_residual_norm_sizes sizes;
    check(sds_residual_norm_bytes(&s.op, &sizes), "sds_residual_norm_bytes");
    const c10::cuda::CUDAGuard guard(r.device());
    // dr, dh, dweight, dbias, dscale, dshift, dgate, dpost_weight
    at::Tensor g[8];
    PyObject* want = a[19];
    if (wanted(want, 0, 8)) g[0] = empty(r.sizes(), r.scalar_type(), r);
    if (wanted(want, 1, 8) && s.h) g[1] = empty(r.sizes(), dn.scalar_type(), r);
    if (wanted(want, 2, 8) && s.op.w_dev) g[2] = empty({s.r.d}, s.w_type, r);
    if (wanted(want, 3, 8) && s.op.b_dev) g[3] = empty({s.r.d}, s.w_type, r);
    const int at[3] = {6, 4, 5};                   // of gate, scale, shift
    for (int k = 0; k < 3; ++k)
      if (wanted(want, at[k], 8) && s.cond[k]) g[at[k]] = empty(s.cond[k]->sizes(), s.c_type, r);
    if (wanted(want, 7, 8) && s.op.post_w_dev) g[7] = empty({s.r.d}, s.w_type, r);
    const int64_t d = s.r.d;
    const sds_residual_norm_grads grads{ptr(g[0]), d, ptr(g[1]), d, ptr(g[2]), ptr(g[3]), ptr(g[7]), ptr(g[6]), ptr(g[4]), ptr(g[5]), d, d, d};
    const at::Tensor ws = workspace(a[20], sizes.backward_bytes, r);
    check(sds_residual_norm_backward(&s.op, dn.data_ptr(), lddn, dout, lddout, r.data_ptr(), s.r.ld, s.h ? s.h->data_ptr() : nullptr, s.ldh,
                                     kept.data_ptr<float>(), &grads, ws.data_ptr(), (size_t)ws.numel(),
                                     c10::cuda::getCurrentCUDAStream(r.get_device()).stream()),
          "sds_residual_norm_backward");
    return tuple({g[0], g[1], g[2], g[3], g[4], g[5], g[6], g[7]});
  });
}

#define SDS_METHOD(name) {#name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(name)), METH_FASTCALL, nullptr}
PyMethodDef methods[] = {SDS_METHOD(layer_norm), SDS_METHOD(layer_norm_backward), SDS_METHOD(gated_ffn),
                         SDS_METHOD(gated_ffn_backward), SDS_METHOD(linear), SDS_METHOD(linear_backward),
                         SDS_METHOD(dropout), SDS_METHOD(residual_norm), SDS_METHOD(residual_norm_backward), {nullptr, nullptr, 0, nullptr}};
PyModuleDef module_def = {PyModuleDef_HEAD_INIT, "_sds_torch", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__sds_torch() { return PyModule_Create(&module_def); }

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

#define SDS_METHOD(name) {#name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(name)), METH_FASTCALL, nullptr}
PyMethodDef methods[] = {SDS_METHOD(layer_norm), SDS_METHOD(layer_norm_backward), SDS_METHOD(gated_ffn),
                         SDS_METHOD(gated_ffn_backward), {nullptr, nullptr, 0, nullptr}};
PyModuleDef module_def = {PyModuleDef_HEAD_INIT, "_sds_torch", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__sds_torch() { return PyModule_Create(&module_def); }

// torch_binding.cpp -- the tensor side of the operators of AAP layers (aecct.py holds their documentation): checks
// of tensors, outputs and workspaces from torch's allocator, and one call of libaecct.  It is C++ because
// the calls are short: a token's norm takes the GPU 4 us, and took 20 us of Python for its four outputs and
// some forty attributes of its tensors; clipping 160 gradients took 197 us of Python.
//
// Streams: without one, a call launches on the current stream.  With one, `_stream_of` (aecct.py) orders it after the
// current stream, where copies are made and outputs allocated, and keeps the tensors for it.
#include <Python.h>

#include <ATen/core/Tensor.h>
#include <ATen/cuda/EmptyTensor.h>
#include <c10/core/GradMode.h>
#include <c10/cuda/CUDAFunctions.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>
#include <torch/csrc/utils/object_ptr.h>

#include <initializer_list>
#include <optional>
#include <string>
#include <vector>

#include "../../include/aecct.h"

namespace {

PyObject *g_stream_of = nullptr, *g_check = nullptr;  // of aecct.py, which keeps them

struct ValueError : std::runtime_error {
  using std::runtime_error::runtime_error;
};
struct PythonError {};  // set already

std::string shape_of(at::IntArrayRef s) {
  std::string t = "(";
  for (size_t i = 0; i < s.size(); ++i) t += std::to_string(s[i]) + (s.size() == 1 ? "," : i + 1 < s.size() ? ", " : "");
  return t + ")";
}

const at::Tensor &tensor(PyObject *o, const char *name) {
  if (!THPVariable_Check(o)) throw ValueError(std::string(name) + " must be a tensor");
  return THPVariable_Unpack(o);
}
const at::Tensor *optional_tensor(PyObject *o, const char *name) { return o == Py_None ? nullptr : &tensor(o, name); }
double number(PyObject *o) {
  const double v = PyFloat_AsDouble(o);
  if (v == -1.0 && PyErr_Occurred()) throw PythonError();
  return v;
}

// the C ABI's number of an element type, -1 for another type
int element(at::ScalarType t) {
  return t == at::kFloat ? AECCT_F32 : t == at::kHalf ? AECCT_F16 : t == at::kBFloat16 ? AECCT_BF16 : -1;
}
at::ScalarType type_of(int element) { return element == AECCT_F32 ? at::kFloat : element == AECCT_F16 ? at::kHalf : at::kBFloat16; }

// an output on a GPU: the allocator's function itself (at::empty finds its way to it in 1.2 us more, of the 5.6 us
// that a token's linear layer took the host)
at::Tensor make(at::IntArrayRef sizes, at::Device on, at::ScalarType type) {
  return at::Tensor(at::detail::empty_cuda(sizes, type, on, std::nullopt));
}
at::Tensor make(at::IntArrayRef sizes, const at::Tensor &like, at::ScalarType type) { return make(sizes, like.device(), type); }

// rows of the last dimension: read where they lie if they are an equal distance apart, else from a contiguous copy
struct Rows {
  at::Tensor t;
  int64_t ld = 0;
  void *p = nullptr;
  Rows() = default;
  explicit Rows(const at::Tensor &x) : t(x), ld(x.size(-1)) {
    if (!x.is_contiguous()) {
      if (x.dim() == 2 && x.stride(1) == 1 && x.stride(0) >= x.size(1)) ld = x.stride(0);
      else t = x.contiguous();
    }
    p = t.data_ptr();
  }
};

void check_like(const char *name, const at::Tensor &t, const at::Tensor &x) {
  if (t.device() != x.device() || t.scalar_type() != x.scalar_type() || t.sizes() != x.sizes())
    throw ValueError(std::string(name) + " must be a tensor of the type, shape " + shape_of(x.sizes()) + " and device of the other rows");
}

// Kernels are launched on the current device, whose SMs their plans count: tensors that lie on another one are refused (launched
// there they would be read across devices, in no order to the work on their own).
void check_current(const at::Device &on) {
  c10::DeviceIndex current = -1;
  if (c10::cuda::GetDevice(&current) != cudaSuccess || current != on.index())
    throw ValueError("the tensors are on " + on.str() + ", which is not the current CUDA device");
}

// The operators record nothing for autograd (int8 codes stand between the norm and the product): where it would
// record, a tensor that requires a gradient is refused, and does not lose it without a word.
void check_no_graph(const char *call, std::initializer_list<const at::Tensor *> tensors) {
  if (!c10::GradMode::is_enabled()) return;
  for (const at::Tensor *t : tensors)
    if (t && t->requires_grad())
      throw ValueError(std::string(call) + " records nothing for autograd: call it under torch.no_grad(), in an autograd.Function, or on detached tensors");
}

// `t` holds rows of a known type on the GPU, and `gain` one float32 for each element of a row
void check_rows(const char *name, const at::Tensor &t, const at::Tensor &gain) {
  if (!t.is_cuda() || element(t.scalar_type()) < 0 || t.dim() < 1)
    throw ValueError(std::string(name) + " must be a float32, float16 or bfloat16 CUDA tensor of rows");
  check_current(t.device());
  if (gain.device() != t.device() || gain.scalar_type() != at::kFloat || gain.dim() != 1 || gain.size(0) != t.size(-1))
    throw ValueError("gain must be a float32 tensor of shape (" + std::to_string(t.size(-1)) + ",) on the rows' device");
}

// the stream to launch on, and with one given, the call's tensors ordered before it and kept for it
void *launch_stream(PyObject *stream, const at::Tensor &on, std::initializer_list<const at::Tensor *> tensors,
                    const std::vector<at::Tensor> *more = nullptr) {
  if (stream == Py_None) return c10::cuda::getCurrentCUDAStream(on.device().index()).stream();
  THPObjectPtr list(PyList_New(0));
  const auto add = [&](const at::Tensor &t) {
    THPObjectPtr o(THPVariable_Wrap(t));
    if (!o || PyList_Append(list.get(), o.get()) < 0) throw PythonError();
  };
  for (const at::Tensor *t : tensors)
    if (t && t->defined()) add(*t);
  if (more)
    for (const at::Tensor &t : *more) add(t);
  THPObjectPtr device(PyLong_FromLong(on.device().index()));
  THPObjectPtr s(PyObject_CallFunctionObjArgs(g_stream_of, stream, device.get(), list.get(), nullptr));
  if (!s) throw PythonError();
  THPObjectPtr raw(PyObject_GetAttrString(s.get(), "cuda_stream"));
  if (!raw) throw PythonError();
  return PyLong_AsVoidPtr(raw.get());
}

void check(int status, const char *what) {
  if (status == AECCT_OK) return;
  THPObjectPtr r(PyObject_CallFunction(g_check, "is", status, what));
  throw PythonError();
}

PyObject *wrap(const at::Tensor &t) {
  if (!t.defined()) Py_RETURN_NONE;
  return THPVariable_Wrap(t);
}
PyObject *tuple(std::initializer_list<at::Tensor> ts) {
  PyObject *r = PyTuple_New(static_cast<Py_ssize_t>(ts.size()));
  Py_ssize_t i = 0;
  for (const at::Tensor &t : ts) PyTuple_SET_ITEM(r, i++, wrap(t));
  return r;
}

// (x, gain, residual, eps, want_values, stream)
PyObject *rms_quant(PyObject *const *a) {
  const at::Tensor &x = tensor(a[0], "x"), &gain = tensor(a[1], "gain");
  const at::Tensor *residual = optional_tensor(a[2], "residual");
  check_rows("x", x, gain);
  if (residual) check_like("residual", *residual, x);
  check_no_graph("rms_quant", {&x, &gain, residual});
  const Rows src(x), res = residual ? Rows(*residual) : Rows();
  const at::Tensor g = gain.contiguous();
  const at::Tensor codes = make(x.sizes(), x, at::kChar), scale = make(x.sizes().slice(0, x.dim() - 1), x, at::kFloat);
  const at::Tensor total = residual ? make(x.sizes(), x, x.scalar_type()) : x;
  const at::Tensor values = a[4] == Py_True ? make(x.sizes(), x, x.scalar_type()) : at::Tensor();
  void *s = launch_stream(a[5], x, {&src.t, &res.t, &g, &codes, &scale, &total, &values});
  check(aecct_rms_quant(src.p, src.ld, res.p, res.ld, static_cast<const float *>(g.data_ptr()), scale.numel(),
                        static_cast<int32_t>(x.size(-1)), element(x.scalar_type()), static_cast<float>(number(a[3])),
                        residual ? total.data_ptr() : nullptr, static_cast<int8_t *>(codes.data_ptr()),
                        static_cast<float *>(scale.data_ptr()), values.defined() ? values.data_ptr() : nullptr, s),
        "aecct_rms_quant");
  return tuple({codes, scale, total, values});
}

// (dy, total, gain, dtotal, eps, stream)
PyObject *rms_quant_backward(PyObject *const *a) {
  const at::Tensor &dy = tensor(a[0], "dy"), &total = tensor(a[1], "total"), &gain = tensor(a[2], "gain");
  const at::Tensor *dtotal = optional_tensor(a[3], "dtotal");
  check_rows("dy", dy, gain);
  check_like("total", total, dy);
  if (dtotal) check_like("dtotal", *dtotal, dy);
  check_no_graph("rms_quant_backward", {&dy, &total, &gain, dtotal});
  const int64_t d = dy.size(-1), rows = d ? dy.numel() / d : 0;
  int64_t bytes = 0;
  check(aecct_rms_quant_backward_workspace(rows, static_cast<int32_t>(d), &bytes), "aecct_rms_quant_backward");
  const Rows g(dy), h(total), dt = dtotal ? Rows(*dtotal) : Rows();
  const at::Tensor gc = gain.contiguous();
  const at::Tensor dx = make(dy.sizes(), dy, dy.scalar_type()), dgain = make({d}, dy, at::kFloat);
  const at::Tensor work = make({bytes}, dy, at::kByte);
  void *s = launch_stream(a[5], dy, {&g.t, &h.t, &dt.t, &gc, &dx, &dgain, &work});
  check(aecct_rms_quant_backward(g.p, g.ld, h.p, h.ld, dt.p, dt.ld, static_cast<const float *>(gc.data_ptr()), rows, static_cast<int32_t>(d),
                                 element(dy.scalar_type()), static_cast<float>(number(a[4])), dx.data_ptr(),
                                 static_cast<float *>(dgain.data_ptr()), work.data_ptr(), bytes, s),
        "aecct_rms_quant_backward");
  return tuple({dx, dgain});
}

struct Linear {
  const at::Tensor &codes, &scale, &packed, &w_scale;
  int64_t M, K, N;
  Linear(PyObject *const *a)
      : codes(tensor(a[0], "codes")), scale(tensor(a[1], "scale")), packed(tensor(a[2], "packed")), w_scale(tensor(a[3], "w_scale")) {
    const at::Device dev = codes.device();
    if (!codes.is_cuda() || codes.scalar_type() != at::kChar || codes.dim() < 1) throw ValueError("codes must be an int8 CUDA tensor of rows");
    check_current(dev);
    K = codes.size(-1);
    const at::IntArrayRef rows = codes.sizes().slice(0, codes.dim() - 1);
    if (scale.device() != dev || scale.scalar_type() != at::kFloat || scale.sizes() != rows)
      throw ValueError("scale must be a float32 tensor of shape " + shape_of(rows) + " on the codes' device");
    if (packed.device() != dev || packed.scalar_type() != at::kByte || !packed.is_contiguous())
      throw ValueError("packed must be a contiguous uint8 tensor on the codes' device");
    if (K < 4 || K % 4 || packed.numel() % (K / 4))
      throw ValueError("rows of " + std::to_string(K) + " codes do not divide weights of " + std::to_string(4 * packed.numel()) + ": K is a multiple of 4");
    if (w_scale.device() != dev || w_scale.scalar_type() != at::kFloat || w_scale.numel() != 1)
      throw ValueError("w_scale must be a float32 tensor of one element on the codes' device");
    M = scale.numel(), N = packed.numel() / (K / 4);
  }
  std::vector<int64_t> out_sizes() const {
    std::vector<int64_t> s(codes.sizes().begin(), codes.sizes().end());
    s.back() = N;
    return s;
  }
};

// the element type that Python names by its number, or an error that says `name`
int32_t element_arg(PyObject *o, const char *name) {
  const long v = o == Py_None ? -1 : PyLong_AsLong(o);
  if (v < 0 || v > AECCT_BF16) throw ValueError(std::string(name) + " must be float32, float16 or bfloat16");
  return static_cast<int32_t>(v);
}

// (codes, scale, packed, w_scale, bias, dtype number, stream)
PyObject *aap_linear(PyObject *const *a) {
  const Linear l(a);
  const at::Tensor *bias = optional_tensor(a[4], "bias");
  const int32_t dtype = element_arg(a[5], "dtype");
  if (bias && (bias->device() != l.codes.device() || bias->scalar_type() != at::kFloat || bias->dim() != 1 || bias->size(0) != l.N))
    throw ValueError("bias must be a float32 tensor of shape (" + std::to_string(l.N) + ",) on the codes' device");
  check_no_graph("aap_linear", {&l.scale, &l.w_scale, bias});
  int64_t bytes = 0;
  check(aecct_aap_linear_workspace(l.M, l.K, l.N, &bytes), "aecct_aap_linear");
  const Rows q(l.codes);
  const at::Tensor scale = l.scale.contiguous(), b = bias ? bias->contiguous() : at::Tensor();
  const at::Tensor y = make(l.out_sizes(), l.codes, type_of(dtype)), work = bytes ? make({bytes}, l.codes, at::kByte) : at::Tensor();
  void *s = launch_stream(a[6], l.codes, {&q.t, &scale, &l.packed, &l.w_scale, &b, &y, &work});
  check(aecct_aap_linear(static_cast<const int8_t *>(q.p), q.ld, static_cast<const float *>(scale.data_ptr()),
                         static_cast<const uint8_t *>(l.packed.data_ptr()), static_cast<const float *>(l.w_scale.data_ptr()),
                         bias ? static_cast<const float *>(b.data_ptr()) : nullptr, l.M, l.K, l.N, dtype, y.data_ptr(),
                         bytes ? work.data_ptr() : nullptr, bytes, s),
        "aecct_aap_linear");
  return wrap(y);
}

// (codes, scale, packed, w_scale, dy, weights' dtype number, want dx, want dw, want db, stream)
PyObject *aap_linear_backward(PyObject *const *a) {
  const Linear l(a);
  const at::Tensor &dy = tensor(a[4], "dy");
  const int32_t wdtype = element_arg(a[5], "weight_dtype");
  const std::vector<int64_t> shape = l.out_sizes();
  if (dy.device() != l.codes.device() || element(dy.scalar_type()) < 0 || dy.sizes() != at::IntArrayRef(shape))
    throw ValueError("dy must be a float32, float16 or bfloat16 tensor of shape " + shape_of(shape) + " on the codes' device");
  const int32_t dtype = element(dy.scalar_type());
  check_no_graph("aap_linear_backward", {&dy, &l.scale, &l.w_scale});
  int64_t bytes = 0;
  check(aecct_aap_linear_backward_workspace(l.M, l.K, l.N, dtype, wdtype, &bytes), "aecct_aap_linear_backward");
  const Rows g(dy), q(l.codes);
  const at::Tensor scale = l.scale.contiguous();
  const bool want[3] = {PyObject_IsTrue(a[6]) == 1, PyObject_IsTrue(a[7]) == 1, PyObject_IsTrue(a[8]) == 1};
  const at::Tensor dx = want[0] ? make(l.codes.sizes(), dy, dy.scalar_type()) : at::Tensor();
  const at::Tensor dw = want[1] ? make({l.N, l.K}, dy, type_of(wdtype)) : at::Tensor();
  const at::Tensor db = want[2] ? make({l.N}, dy, at::kFloat) : at::Tensor();
  const at::Tensor work = bytes ? make({bytes}, dy, at::kByte) : at::Tensor();
  void *s = launch_stream(a[9], dy, {&g.t, &q.t, &scale, &l.packed, &l.w_scale, &dx, &dw, &db, &work});
  check(aecct_aap_linear_backward(g.p, g.ld, static_cast<const int8_t *>(q.p), q.ld, static_cast<const float *>(scale.data_ptr()),
                                  static_cast<const uint8_t *>(l.packed.data_ptr()), static_cast<const float *>(l.w_scale.data_ptr()),
                                  l.M, l.K, l.N, dtype, wdtype, want[0] ? dx.data_ptr() : nullptr, want[1] ? dw.data_ptr() : nullptr,
                                  want[2] ? static_cast<float *>(db.data_ptr()) : nullptr, bytes ? work.data_ptr() : nullptr, bytes, s),
        "aecct_aap_linear_backward");
  return tuple({dx, dw, db});
}

// (list of gradients, max_norm, eps, list of outputs or None, current device's index where there are no gradients, stream)
PyObject *clip_gradients(PyObject *const *a) {
  THPObjectPtr grads(PySequence_Fast(a[0], "grads must be a sequence of tensors"));
  if (!grads) throw PythonError();
  THPObjectPtr outs(a[3] == Py_None ? nullptr : PySequence_Fast(a[3], "out must be a sequence of tensors"));
  if (a[3] != Py_None && !outs) throw PythonError();
  const Py_ssize_t n = PySequence_Fast_GET_SIZE(grads.get());
  if (outs && PySequence_Fast_GET_SIZE(outs.get()) != n) throw ValueError("out must have " + std::to_string(n) + " tensors");
  std::vector<const void *> src(n);
  std::vector<void *> dst(n);
  std::vector<int64_t> len(n);
  std::vector<int32_t> type(n);
  std::vector<at::Tensor> kept;
  at::Device dev(at::kCUDA, static_cast<at::DeviceIndex>(PyLong_AsLong(a[4])));
  for (Py_ssize_t j = 0; j < n; ++j) {
    const at::Tensor &g = tensor(PySequence_Fast_GET_ITEM(grads.get(), j), "a gradient");
    const at::Tensor &o = outs ? tensor(PySequence_Fast_GET_ITEM(outs.get(), j), "an output") : g;
    if (j == 0) {
      dev = g.device();
      if (!g.is_cuda()) throw ValueError("clip_gradients takes CUDA tensors");
      check_current(dev);
    }
    if ((type[j] = element(g.scalar_type())) < 0 || g.device() != dev || !g.is_contiguous())
      throw ValueError("gradients must be contiguous float32, float16 or bfloat16 tensors on one device");
    if (outs && (o.scalar_type() != g.scalar_type() || o.sizes() != g.sizes() || o.device() != dev || !o.is_contiguous()))
      throw ValueError("out must hold contiguous tensors like the gradients");
    src[j] = g.data_ptr(), dst[j] = o.data_ptr(), len[j] = g.numel();
    if (a[5] != Py_None) {
      kept.push_back(g);
      if (outs) kept.push_back(o);
    }
  }
  int64_t bytes = 0;
  check(aecct_clip_workspace(static_cast<int32_t>(n), &bytes), "aecct_clip_gradients");
  const at::Tensor norm = make({}, dev, at::kFloat), work = make({bytes}, dev, at::kByte);
  void *s = launch_stream(a[5], norm, {&norm, &work}, &kept);
  check(aecct_clip_gradients(static_cast<int32_t>(n), src.data(), len.data(), type.data(), dst.data(), static_cast<float>(number(a[1])),
                             static_cast<float>(number(a[2])), static_cast<float *>(norm.data_ptr()), work.data_ptr(), bytes, s),
        "aecct_clip_gradients");
  for (Py_ssize_t j = 0; j < n; ++j) {  // (written in place, as autograd counts it)
    const at::Tensor &o = THPVariable_Unpack(PySequence_Fast_GET_ITEM(outs ? outs.get() : grads.get(), j));
    if (!o.is_inference()) o.unsafeGetTensorImpl()->bump_version();
  }
  return wrap(norm);
}

template <PyObject *(*F)(PyObject *const *), Py_ssize_t N>
PyObject *entry(PyObject *, PyObject *const *args, Py_ssize_t n) {
  if (n != N) {
    PyErr_SetString(PyExc_TypeError, "wrong number of arguments");
    return nullptr;
  }
  HANDLE_TH_ERRORS
  try {
    return F(args);
  } catch (const ValueError &e) {
    PyErr_SetString(PyExc_ValueError, e.what());
    return nullptr;
  } catch (const PythonError &) {
    return nullptr;
  }
  END_HANDLE_TH_ERRORS
}

// (_stream_of, _check)
PyObject *setup(PyObject *const *a) {
  Py_INCREF(a[0]), Py_INCREF(a[1]);
  g_stream_of = a[0], g_check = a[1];
  Py_RETURN_NONE;
}

template <PyObject *(*F)(PyObject *const *), Py_ssize_t N>
PyMethodDef method(const char *name) {
  return {name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(&entry<F, N>)), METH_FASTCALL, nullptr};
}
PyMethodDef g_methods[] = {method<setup, 2>("setup"),
                           method<rms_quant, 6>("rms_quant"),
                           method<rms_quant_backward, 6>("rms_quant_backward"),
                           method<aap_linear, 7>("aap_linear"),
                           method<aap_linear_backward, 10>("aap_linear_backward"),
                           method<clip_gradients, 6>("clip_gradients"),
                           {nullptr, nullptr, 0, nullptr}};
PyModuleDef g_module = {PyModuleDef_HEAD_INIT, "aecct_torch", nullptr, -1, g_methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit_aecct_torch() { return PyModule_Create(&g_module); }

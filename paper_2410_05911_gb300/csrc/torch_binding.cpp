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
#include <c10/core/AutogradState.h>
#include <c10/core/GradMode.h>
#include <c10/cuda/CUDAFunctions.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>
#include <torch/csrc/utils/object_ptr.h>

#include <climits>
#include <cmath>
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
// record, a tensor that requires a gradient is refused, and does not lose it without a word.  Nor does one with a tangent (forward mode, which
// torch.no_grad() leaves on and an autograd.Function turns off) lose that.
void check_no_graph(const char *call, std::initializer_list<const at::Tensor *> tensors) {
  const bool reverse = c10::GradMode::is_enabled(), forward = c10::AutogradState::get_tls_state().get_fw_grad_mode();
  if (!reverse && !forward) return;
  for (const at::Tensor *t : tensors) {
    if (!t || !t->defined()) continue;
    if (reverse && t->requires_grad())
      throw ValueError(std::string(call) + " records nothing for autograd: call it under torch.no_grad(), in an autograd.Function, or on detached tensors");
    if (forward && t->_fw_grad(0).defined())
      throw ValueError(std::string(call) + " carries no tangents of forward mode: call it in an autograd.Function, or on the primal of a dual tensor");
  }
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

// ------------------------------------------------------------------------------------------
// serving a token at a time
// ------------------------------------------------------------------------------------------
int cache_element(at::ScalarType t) { return t == at::kChar ? AECCT_I8 : t == at::kFloat ? -1 : element(t); }

// a KVCache: its four tensors, checked
struct Cache {
  at::Tensor k, v, k_scale, v_scale;
  aecct_kv_cache c = {};
  explicit Cache(PyObject *o) {
    if (!PyTuple_Check(o) || PyTuple_GET_SIZE(o) != 4) throw ValueError("cache must be a KVCache");
    k = tensor(PyTuple_GET_ITEM(o, 0), "cache.k"), v = tensor(PyTuple_GET_ITEM(o, 1), "cache.v");
    if (!k.is_cuda() || cache_element(k.scalar_type()) < 0 || k.dim() != 4)
      throw ValueError("cache.k must be an int8, float16 or bfloat16 CUDA tensor [pages, heads, page_size, head_dim]");
    check_current(k.device());
    const auto s = k.sizes();
    if (v.device() != k.device() || v.scalar_type() != k.scalar_type() || v.sizes() != s) throw ValueError("cache.v must be a tensor like cache.k");
    c.dtype = cache_element(k.scalar_type());
    c.ld = row_stride(k);
    if (row_stride(v) != c.ld) throw ValueError("cache.v must be laid out like cache.k");
    const bool scaled = c.dtype == AECCT_I8;
    for (int i = 2; i < 4; ++i) {
      const at::Tensor *t = optional_tensor(PyTuple_GET_ITEM(o, i), "a cache's scale");
      if (!scaled && t) throw ValueError("a cache of 16-bit rows has no scales");
      if (scaled && (!t || t->device() != k.device() || t->scalar_type() != at::kFloat || t->sizes() != s.slice(0, 3) || !t->is_contiguous()))
        throw ValueError("an int8 cache's scales must be contiguous float32 tensors of shape " + shape_of(s.slice(0, 3)));
      if (scaled) (i == 2 ? k_scale : v_scale) = *t;
    }
    c.k = k.data_ptr(), c.v = v.data_ptr();
    if (scaled) c.k_scale = static_cast<float *>(k_scale.data_ptr()), c.v_scale = static_cast<float *>(v_scale.data_ptr());
    for (int i = 1; i < 4; ++i)
      if (s[i] >= (1 << 20)) throw ValueError("cache.k has a size that is too large");
    c.pages = s[0], c.heads = static_cast<int32_t>(s[1]), c.page_size = static_cast<int32_t>(s[2]), c.head_dim = static_cast<int32_t>(s[3]);
  }

 private:
  // elements from one row to the next: pages, heads and places follow one another without a gap
  static int32_t row_stride(const at::Tensor &t) {
    const auto s = t.sizes(), st = t.strides();
    const int64_t size = t.element_size();
    int64_t ld = s[2] > 1 ? st[2] : s[1] > 1 ? st[1] : s[0] > 1 ? st[0] : (s[3] * size + 15) / 16 * 16 / size;
    if (ld > (1 << 20) || ld < s[3] || ld * size % 16 || (t.numel() > 0 && (reinterpret_cast<uintptr_t>(t.data_ptr()) & 15u)) || (s[3] > 1 && st[3] != 1) ||
        (s[1] > 1 && st[1] != s[2] * ld) || (s[0] > 1 && st[0] != s[1] * s[2] * ld))
      throw ValueError("a cache's rows must lie an equal multiple of 16 bytes apart, as kv_cache makes them");
    return static_cast<int32_t>(ld);
  }
};

at::Tensor int_array(PyObject *o, const char *name, const at::Device &on, int64_t n) {
  const at::Tensor &t = tensor(o, name);
  if (t.device() != on || t.scalar_type() != at::kInt || t.dim() != 1 || t.size(0) != n)
    throw ValueError(std::string(name) + " must be an int32 tensor of shape (" + std::to_string(n) + ",) on the cache's device");
  return t.contiguous();
}

// table and lengths
struct Sequences {
  at::Tensor table, lengths;
  aecct_kv_sequences s = {};
  Sequences(PyObject *t, PyObject *l, const at::Device &on) {
    table = tensor(t, "table");
    if (table.device() != on || table.scalar_type() != at::kInt || table.dim() != 2 || table.size(0) > INT32_MAX || table.size(1) > INT32_MAX)
      throw ValueError("table must be an int32 tensor [batch, columns] on the cache's device");
    lengths = int_array(l, "lengths", on, table.size(0));
    const Rows r(table);
    table = r.t;
    s.table = static_cast<const int32_t *>(r.p), s.ldt = r.ld, s.lengths = static_cast<const int32_t *>(lengths.data_ptr());
    s.batch = static_cast<int32_t>(table.size(0)), s.columns = static_cast<int32_t>(table.size(1));
  }
};

// [tokens][heads][dim], read where it lies if the elements of a row do
struct Heads {
  at::Tensor t;
  int64_t row, head;
  explicit Heads(const at::Tensor &x) : t(x.size(2) > 1 && x.stride(2) != 1 ? x.contiguous() : x), row(t.stride(0)), head(t.stride(1)) {}
};

// the arrays after the first, with the check that they are like it
const at::Tensor &heads_of(PyObject *o, const char *name, const Cache &cache, bool same_heads) {
  const at::Tensor &t = tensor(o, name);
  if (t.device() != cache.k.device() || element(t.scalar_type()) < 0 || t.dim() != 3 || t.size(2) != cache.c.head_dim ||
      (same_heads && t.size(1) != cache.c.heads))
    throw ValueError(std::string(name) + " must be a float32, float16 or bfloat16 tensor [tokens, " + (same_heads ? "" : "q_") + "heads, head_dim] on the cache's device");
  if (cache.c.dtype != AECCT_I8 && cache.c.dtype != element(t.scalar_type())) throw ValueError(std::string(name) + " must have the type of a 16-bit cache");
  return t;
}

// (k, v, cache, table, lengths, rows, stream)
PyObject *kv_append(PyObject *const *a) {
  const Cache cache(a[2]);
  const at::Device on = cache.k.device();
  const at::Tensor &k = heads_of(a[0], "k", cache, true), &v = heads_of(a[1], "v", cache, true);
  check_like("v", v, k);
  const Sequences seqs(a[3], a[4], on);
  const int64_t total = k.size(0);
  const at::Tensor rows = a[5] == Py_None ? at::Tensor() : int_array(a[5], "rows", on, int64_t(seqs.s.batch) + 1);
  if (!rows.defined() && total != seqs.s.batch) throw ValueError("without rows, k has one token for each of " + std::to_string(seqs.s.batch) + " sequences");
  check_no_graph("kv_append", {&k, &v, &cache.k, &cache.v, &cache.k_scale, &cache.v_scale});
  const Heads kh(k), vh(v);
  void *s = launch_stream(a[6], cache.k, {&kh.t, &vh.t, &cache.k, &cache.v, &cache.k_scale, &cache.v_scale, &seqs.table, &seqs.lengths, &rows});
  check(aecct_kv_append(&cache.c, &seqs.s, rows.defined() ? static_cast<const int32_t *>(rows.data_ptr()) : nullptr, total, kh.t.data_ptr(), kh.row, kh.head,
                        vh.t.data_ptr(), vh.row, vh.head, element(k.scalar_type()), s),
        "aecct_kv_append");
  for (const at::Tensor *t : {&cache.k, &cache.v, &cache.k_scale, &cache.v_scale})  // (written in place, as autograd counts it)
    if (t->defined() && !t->is_inference()) t->unsafeGetTensorImpl()->bump_version();
  Py_RETURN_NONE;
}

// (cache, table, lengths, rows, total, dtype number, stream)
PyObject *kv_read(PyObject *const *a) {
  const Cache cache(a[0]);
  const at::Device on = cache.k.device();
  const Sequences seqs(a[1], a[2], on);
  const at::Tensor rows = a[3] == Py_None ? at::Tensor() : int_array(a[3], "rows", on, int64_t(seqs.s.batch) + 1);
  const int64_t total = PyLong_AsLongLong(a[4]);
  if (total == -1 && PyErr_Occurred()) throw PythonError();
  if (total < 0) throw ValueError("total must not be negative");
  if (!rows.defined() && total != seqs.s.batch) throw ValueError("without rows, there is one token for each of " + std::to_string(seqs.s.batch) + " sequences");
  const int32_t dtype = element_arg(a[5], "dtype");
  check_no_graph("kv_read", {&cache.k, &cache.v, &cache.k_scale, &cache.v_scale});
  const at::Tensor k = make({total, cache.c.heads, cache.c.head_dim}, on, type_of(dtype)), v = make({total, cache.c.heads, cache.c.head_dim}, on, type_of(dtype));
  void *s = launch_stream(a[6], cache.k, {&k, &v, &cache.k, &cache.v, &cache.k_scale, &cache.v_scale, &seqs.table, &seqs.lengths, &rows});
  check(aecct_kv_read(&cache.c, &seqs.s, rows.defined() ? static_cast<const int32_t *>(rows.data_ptr()) : nullptr, total, k.data_ptr(), v.data_ptr(), dtype, s),
        "aecct_kv_read");
  return tuple({k, v});
}

// (q, cache, table, lengths, first, scale, want_lse, stream)
PyObject *paged_attention(PyObject *const *a) {
  const Cache cache(a[1]);
  const at::Device on = cache.k.device();
  const at::Tensor &q = heads_of(a[0], "q", cache, false);
  const Sequences seqs(a[2], a[3], on);
  if (q.size(0) != seqs.s.batch) throw ValueError("q must have a token for each of " + std::to_string(seqs.s.batch) + " sequences");
  if (cache.c.heads < 1 || q.size(1) < 1 || q.size(1) % cache.c.heads || q.size(1) >= (1 << 20))
    throw ValueError("the heads of q must be a multiple of the cache's " + std::to_string(cache.c.heads));
  const at::Tensor first = a[4] == Py_None ? at::Tensor() : int_array(a[4], "first", on, seqs.s.batch);
  const double scale = a[5] == Py_None ? 1.0 / std::sqrt(static_cast<double>(cache.c.head_dim)) : number(a[5]);
  check_no_graph("paged_attention", {&q, &cache.k, &cache.v, &cache.k_scale, &cache.v_scale});
  const int32_t q_heads = static_cast<int32_t>(q.size(1)), dtype = element(q.scalar_type());
  int64_t bytes = 0;
  check(aecct_paged_attention_workspace(seqs.s.batch, q_heads, cache.c.heads, cache.c.head_dim, dtype, cache.c.dtype, &bytes), "aecct_paged_attention");
  const Heads qh(q);
  const at::Tensor out = make(q.sizes(), on, q.scalar_type()), lse = a[6] == Py_True ? make({seqs.s.batch, q_heads}, on, at::kFloat) : at::Tensor();
  const at::Tensor work = bytes ? make({bytes}, on, at::kByte) : at::Tensor();
  void *s = launch_stream(a[7], q, {&qh.t, &cache.k, &cache.v, &cache.k_scale, &cache.v_scale, &seqs.table, &seqs.lengths, &first, &out, &lse, &work});
  check(aecct_paged_attention(&cache.c, &seqs.s, first.defined() ? static_cast<const int32_t *>(first.data_ptr()) : nullptr, qh.t.data_ptr(), qh.row, qh.head,
                              q_heads, dtype, static_cast<float>(scale), out.data_ptr(), lse.defined() ? static_cast<float *>(lse.data_ptr()) : nullptr,
                              bytes ? work.data_ptr() : nullptr, bytes, s),
        "aecct_paged_attention");
  return tuple({out, lse});
}

// a setting of sample: a tensor with one for each row, or a number
at::Tensor setting(PyObject *o, const char *name, const at::Tensor &logits, at::ScalarType type, double *all) {
  if (!THPVariable_Check(o)) {
    *all = number(o);
    return at::Tensor();
  }
  const at::Tensor &t = THPVariable_Unpack(o);
  const at::IntArrayRef rows = logits.sizes().slice(0, logits.dim() - 1);
  if (t.device() != logits.device() || t.scalar_type() != type || t.sizes() != rows)
    throw ValueError(std::string(name) + " must be a number, or " + (type == at::kInt ? "an int32" : "a float32") + " tensor of shape " + shape_of(rows) +
                     " on the logits' device");
  return t.contiguous();
}

// (logits, u, temperature, top_k, top_p, min_p, stream)
PyObject *sample(PyObject *const *a) {
  const at::Tensor &logits = tensor(a[0], "logits"), &u = tensor(a[1], "u");
  if (!logits.is_cuda() || element(logits.scalar_type()) < 0 || logits.dim() < 1)
    throw ValueError("logits must be a float32, float16 or bfloat16 CUDA tensor of rows");
  check_current(logits.device());
  const at::IntArrayRef shape = logits.sizes().slice(0, logits.dim() - 1);
  if (u.device() != logits.device() || u.scalar_type() != at::kFloat || u.sizes() != shape)
    throw ValueError("u must be a float32 tensor of shape " + shape_of(shape) + " on the logits' device");
  if (logits.size(-1) > INT32_MAX) throw ValueError("the rows of logits are too long");
  double t = 0, k = 0, p = 0, m = 0;
  const at::Tensor ts = setting(a[2], "temperature", logits, at::kFloat, &t), ks = setting(a[3], "top_k", logits, at::kInt, &k);
  const at::Tensor ps = setting(a[4], "top_p", logits, at::kFloat, &p), ms = setting(a[5], "min_p", logits, at::kFloat, &m);
  if (!(k >= 0) || k != std::floor(k)) throw ValueError("top_k must be a whole number that is not negative");
  check_no_graph("sample", {&logits, &u, &ts, &ps, &ms});
  const Rows x(logits);
  const at::Tensor uc = u.contiguous(), tokens = make(shape, logits, at::kLong);
  const auto floats = [](const at::Tensor &v) { return v.defined() ? static_cast<const float *>(v.data_ptr()) : nullptr; };
  aecct_sample_settings set = {};
  set.temperature_dev = floats(ts), set.top_p_dev = floats(ps), set.min_p_dev = floats(ms);
  set.top_k_dev = ks.defined() ? static_cast<const int32_t *>(ks.data_ptr()) : nullptr;
  set.temperature = static_cast<float>(t), set.top_p = static_cast<float>(p), set.min_p = static_cast<float>(m);
  set.top_k = k >= INT32_MAX ? 0 : static_cast<int32_t>(k);
  void *s = launch_stream(a[6], logits, {&x.t, &uc, &ts, &ks, &ps, &ms, &tokens});
  check(aecct_sample(x.p, x.ld, uc.numel(), static_cast<int32_t>(logits.size(-1)), element(logits.scalar_type()), static_cast<const float *>(uc.data_ptr()), &set,
                     static_cast<int64_t *>(tokens.data_ptr()), s),
        "aecct_sample");
  return wrap(tokens);
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
                           method<kv_append, 7>("kv_append"),
                           method<kv_read, 7>("kv_read"),
                           method<paged_attention, 8>("paged_attention"),
                           method<sample, 7>("sample"),
                           {nullptr, nullptr, 0, nullptr}};
PyModuleDef g_module = {PyModuleDef_HEAD_INIT, "aecct_torch", nullptr, -1, g_methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit_aecct_torch() { return PyModule_Create(&g_module); }
